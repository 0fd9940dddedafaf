// fcp_cache_attn_shared: attention over the paged 8-bit cache where the sequences of a group have a common beginning.
//
// softmax over a sequence's tokens is put together from two parts: the common beginning, which all rows of the group see whole, and the sequence's own rest.  The group's rows are next
// to each other, so the common part is attention of many rows over one run of keys: its bytes are read once for the group instead of once for every sequence, and where one token of a
// sequence alone would leave the matrix units idle, a group's rows fill their tiles.  Partial results (sums, maximum, sum of exponentials) meet in the last launch.
//   * All common parts are one line of tiles, all own parts another (csrc/fcp_cache_attn.h).  Every block places the parts by itself where they are few; else a launch of one block does.
//   * One launch works both lines, the common one with the bodies for few or for many rows, as the rows of a group are on average; a wave works an own part alone.  Where sequences have more than 16 rows
//     for a KV head on average each line has a launch of its own.
//   * A wave for each row joins the pieces of its two items, whose places their workers left for it.
// 64 samples of a prompt of up to 16384 tokens, e4m3, 32 query heads over 8 KV heads of 128: 59 us, 52 and 9.4 of them the launches under a
// profiler, fcp_cache_attn 174; the products of the common part would take a large product's rate 14 us (21 with probabilities in two parts), the blocks begin them 10 us after the launch does (places 3.4, own
// parts and the first loads the rest), and partial results are 34 MB.  16 prompts of up to 8000 tokens, 8 beams each, int8: 50 us, 44 and 6.6 under a profiler, where reading every key once takes 24.
#include "fcp_cache_few.h"
#include "fcp_cache_many.h"

namespace fcp {
namespace {

enum { kCommon = 0, kOwn = 1 };

// A run of cached tokens and the rows that attend over it, as the tables of parts hold it.
struct Entry {
  int32_t row0, rows;                  // rows of q, tokens; rows = 0: nothing to do
  int32_t other;                       // common: the sequence whose pages are read; own: the common part of the rows, or -1
  int32_t len;                         // common: tokens; own: tokens of the sequence, common ones included
};
static_assert(sizeof(Entry) == 16, "four words");

// In LDS or in scratch: the parts; the places of those before on their line, of all, and whether items are one place each (kWhole) or tiles and a lead.
struct Tables {
  Entry* common;
  Entry* own;
  int32_t* before_common;
  int32_t* before_own;
  __device__ Entry* e(int kind) const { return kind == kCommon ? common : own; }
  __device__ int32_t* before(int kind) const { return kind == kCommon ? before_common : before_own; }
};

// Where the pieces of a row's item lie: slots of blocks (waves) first, first + 1, ..; n = 1: in `whole`.  lr: its row in a slot.  common: own parts: the row has a common part too (else what the
// common part's worker noted for the row does not count).
struct RowPieces { int32_t first, n, lr, common; };

struct SharedArgs {
  CacheView c;
  SeqView s;
  const int32_t* groups;
  const int32_t* shared_len;
  int32_t n_groups;
  const __bf16* q;
  int64_t q_row;
  int32_t hq, group;
  float scale;
  __bf16* o;
  float* lse;
  Tables tables;                       // in scratch
  struct RowPieces* pieces[2];         // [tq * hq], of all rows of sequences
  int32_t log_rows[2], log_sharers[2]; // rows of an item; blocks, or waves, that may share a line
  float* slots[2];                     // two per block: pieces of divided items
  int32_t waves;                       // own parts: a wave works an item, else a block
  int32_t local;                       // blocks place the parts themselves
  float* whole[2];                     // items in one piece: [tq * hq][D + 2], sums, maximum, sum of exponentials
  __device__ int32_t count(int kind) const { return kind == kCommon ? n_groups : s.n_seqs; }
};

// A part, whole: its rows, its pages (those of the table's row from page0 on), tokens; row i sees those up to first_seen + each * i.
struct Part { int32_t row0, rows, seq, page0, len, first_seen, each, common; };       // common: own parts: their rows have a common part
__device__ inline Part part_of(const SharedArgs& a, const Tables& t, int kind, int i) {
  const Entry x = t.e(kind)[i];
  if (kind == kCommon) return {x.row0, x.rows, x.other, 0, x.len, x.len - 1, 0, 0};
  const int32_t shared = x.other >= 0 ? t.common[x.other].len : 0, len = x.len - shared;
  return {x.row0, x.rows, i, shared >> a.c.log_page, len, len - x.rows, 1, shared > 0};
}
__device__ inline int32_t places_of_item(const Part& p, bool whole) { return whole ? 1 : places_of<kItemLead>(p.len); }
__device__ inline int32_t row_blocks_of(const SharedArgs& a, const Part& p, int kind) { return ((p.rows * a.group - 1) >> a.log_rows[kind]) + 1; }
__device__ inline int32_t places_of_part(const SharedArgs& a, const Part& p, int kind, bool whole) { return p.rows == 0 ? 0 : a.c.hkv * row_blocks_of(a, p, kind) * places_of_item(p, whole); }

// Own parts up to this long are not divided, where all are.  4 / 8 / 16 tiles: 64 of a group with 600 own tokens 67.9 / 68.3 / 68.1 us, with 300 62.8 / 59.8 / 59.9, 8 with 1000 36.5 / 36.4 / 51.6.
constexpr int kWholeLen = 8 * kTile;
constexpr int kSharers = kWaves * kBlocks;       // waves that share the line of own parts
constexpr int kLocal = 256;            // parts that a block places itself: one a thread

// Places 0 .. total - 1 in `n` shares that differ by one place at most.
struct Even {
  int32_t total, n, log_most;          // n: up to 2^log_most
  __device__ int32_t each() const { return n >> log_most ? total >> log_most : (int32_t)((uint32_t)total / (uint32_t)n); }
  __device__ int32_t begin(int32_t i) const {
    const int32_t q = each();
    return i * q + min(i, total - n * q);
  }
  __device__ int32_t owner(int32_t x) const {
    const int32_t q = each(), r = total - n * q, first = r * (q + 1);
    return x < first ? (int32_t)((uint32_t)x / (uint32_t)(q + 1)) : r + (int32_t)((uint32_t)(x - first) / (uint32_t)q);
  }
};
// A line and its shares: a share has a few places at least, where items are one place each one.
struct Shares {
  Even even;
  bool whole;
};
__device__ inline Shares shares_of(const SharedArgs& a, const Tables& t, int kind) {
  const int32_t* const ends = t.before(kind) + a.count(kind);
  const int32_t total = __builtin_amdgcn_readfirstlane(ends[0]);
  const bool whole = __builtin_amdgcn_readfirstlane(ends[1]);
  return {{total, min(1 << a.log_sharers[kind], whole ? total : (total + kLeastTiles - 1) / kLeastTiles), a.log_sharers[kind]}, whole};
}
// Shares of the common line go to the blocks from the last one on, those of the own line from the first: where there are few, different blocks have them.
__device__ inline int share_of_block(const SharedArgs& a, int kind) { return kind == kCommon && a.waves ? kBlocks - 1 - (int)blockIdx.x : (int)blockIdx.x; }

// The common parts from the groups and the own parts' entries; these learn their group.
struct Group { int32_t lo, hi, said; };
// What every row of a group sees, at most `said`, its first sequence, its first row and the one behind its last, its sequences: of some of its sequences.  Those without rows do not count, nor do those
// with a row that does not see a page before the new ones (a beam that has just begun): these are worked by themselves, and do not keep the others from what they have in common.  Where the rows of
// such a sequence lie between the others' they are worked with them, and nobody looks at what comes out.
struct Seen { int32_t least, first, row0, end, seqs; };
__device__ inline Seen look_at(const Tables& t, const Group& x, int g, int sub, int lanes, int page) {
  Seen r = {max(x.said, 0), INT32_MAX, INT32_MAX, 0, 0};
  for (int s = x.lo + sub; s < x.hi; s += lanes) {
    const Entry y = t.own[s];
    if (y.rows > 0 && y.len - y.rows >= page) {
      t.own[s].other = g;
      r.least = min(r.least, y.len - y.rows);
      r.first = min(r.first, s);
      r.row0 = min(r.row0, y.row0);
      r.end = max(r.end, y.row0 + y.rows);
      ++r.seqs;
    }
  }
  return r;
}
__device__ inline Entry common_of(const Seen& x, int page) {
  const int32_t shared = x.seqs < 2 ? 0 : x.least & ~(page - 1);
  return {x.row0, shared ? x.end - x.row0 : 0, x.first, shared};
}
template <int Threads, class F>
__device__ inline void place_groups(const SharedArgs& a, const Tables& t, F group) {
  if (a.n_groups <= Threads / 64) {                                     // a wave a group (300 sequences of one group: 52 us, 58 with eight lanes)
    const int g = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (g >= a.n_groups) return;
    Seen x = look_at(t, group(g), g, lane, 64, a.c.page);
    auto least_of = [](int32_t v) { return INT32_MAX - wave_max(INT32_MAX - v); };
    auto sum_of = [](int32_t v) { return __builtin_amdgcn_readlane(wave_prefix_sum(v), 63); };
    x = {least_of(x.least), least_of(x.first), least_of(x.row0), wave_max(x.end), sum_of(x.seqs)};
    if (lane == 0) t.common[g] = common_of(x, a.c.page);
    return;
  }
  for (int g0 = 0; g0 < a.n_groups; g0 += Threads / 8) {                // eight lanes a group
    const int g = g0 + (int)threadIdx.x / 8, sub = threadIdx.x % 8;
    Seen x = look_at(t, g < a.n_groups ? group(g) : Group{0, 0, 0}, g, sub, 8, a.c.page);
#pragma unroll
    for (int d = 1; d < 8; d *= 2)
      x = {min(x.least, __shfl_xor(x.least, d)), min(x.first, __shfl_xor(x.first, d)), min(x.row0, __shfl_xor(x.row0, d)), max(x.end, __shfl_xor(x.end, d)), x.seqs + __shfl_xor(x.seqs, d)};
    if (g < a.n_groups && sub == 0) t.common[g] = common_of(x, a.c.page);
  }
}

// Fills the tables.  Where cu_seqlens or groups fall, or groups name sequences that are not there, there are no places.
template <int Threads>
__device__ inline void place_parts(const SharedArgs& a, const Tables& t) {
  __shared__ int32_t sums[Threads / 64], bad, longest;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) bad = longest = 0;
  __syncthreads();
  bool falls = false;
  for (int s = threadIdx.x; s < a.s.n_seqs; s += Threads) {
    falls |= a.s.cu[s + 1] < a.s.cu[s];
    const SeqSizes z = seq_sizes(a.s, s, a.c.page);
    t.own[s] = {z.row0, z.n, -1, z.len};
  }
  for (int g = threadIdx.x; g < a.n_groups; g += Threads) falls |= a.groups[g] < 0 || a.groups[g + 1] < a.groups[g] || a.groups[g + 1] > a.s.n_seqs;
  if (falls) bad = 1;
  __syncthreads();
  if (!bad)
    place_groups<Threads>(a, t, [&](int g) { return Group{a.groups[g], a.groups[g + 1], a.shared_len[g]}; });
  __syncthreads();
  int32_t most = 0;
  if (!bad)
    for (int s = threadIdx.x; s < a.s.n_seqs; s += Threads) {
      const Part p = part_of(a, t, kOwn, s);
      if (p.rows > 0) most = max(most, p.len);
    }
  most = wave_max(most);
  if (lane == 0) atomicMax(&longest, most);
  __syncthreads();
  for (int kind = 0; kind < 2; ++kind) {
    const int n = a.count(kind);
    const bool whole = kind == kOwn && a.waves && longest <= kWholeLen;
    int32_t total = 0;
    for (int i0 = 0; i0 < n; i0 += Threads) {
      const int i = i0 + threadIdx.x;
      const int32_t mine = i < n && !bad ? places_of_part(a, part_of(a, t, kind, i), kind, whole) : 0, upto = wave_prefix_sum(mine);
      if (lane == 63) sums[wave] = upto;
      __syncthreads();
      int32_t at = total + upto - mine;
      for (int w = 0; w < Threads / 64; ++w) {
        at += w < wave ? sums[w] : 0;
        total += sums[w];
      }
      if (i < n) t.before(kind)[i] = at;
      __syncthreads();
    }
    if (threadIdx.x == 0) t.before(kind)[n] = total, t.before(kind)[n + 1] = whole;
  }
}

constexpr int kPartThreads = 1024;
__global__ __launch_bounds__(kPartThreads) void parts_kernel(SharedArgs a) { place_parts<kPartThreads>(a, a.tables); }

// The same by every block of a line's launch, where there are up to kLocal sequences: a thread looks at a sequence and at a group, and everything is asked for at once.  (A launch of one block takes
// 5 to 7 us.)  The join learns from the first block whether there is anything to do.
struct LocalTables { Entry e[2][kLocal]; int32_t before[2][kLocal + 2]; };
__device__ inline Tables tables_of(const SharedArgs& a, LocalTables& own) {
  if (!a.local) return a.tables;
  __shared__ int32_t sums[3][4], longest[4], bad[4];
  const Tables t = {own.e[0], own.e[1], own.before[0], own.before[1]};
  const int i = threadIdx.x, lane = i & 63, wave = i >> 6;
  const bool is_seq = i < a.s.n_seqs, is_group = i < a.n_groups;
  const SeqSizes z = is_seq ? seq_sizes(a.s, i, a.c.page) : SeqSizes{};
  bool falls = is_seq && a.s.cu[i + 1] < a.s.cu[i];
  const int lo = is_group ? a.groups[i] : 0, hi = is_group ? a.groups[i + 1] : 0, said = is_group ? a.shared_len[i] : 0;
  falls |= lo < 0 || hi < lo || hi > a.s.n_seqs;
  if (is_seq) t.own[i] = {z.row0, z.n, -1, z.len};
  if (is_group) t.common[i] = {lo, hi, said, 0};
  falls = __ballot(falls);
  if (lane == 0) bad[wave] = falls;
  __syncthreads();
  const bool none = bad[0] | bad[1] | bad[2] | bad[3];
  if (!none) place_groups<kLocal>(a, t, [&](int g) { const Entry x = t.common[g]; return Group{x.row0, x.rows, x.other}; });
  __syncthreads();
  // places of the thread's sequence if items are one place each, and if they are not; of its group
  int32_t places[3] = {}, upto[3], most = 0;
  if (is_seq && !none) {
    const Part p = part_of(a, t, kOwn, i);
    places[0] = places_of_part(a, p, kOwn, false);
    places[1] = places_of_part(a, p, kOwn, true);
    most = p.rows > 0 ? p.len : 0;
  }
  if (is_group && !none) places[2] = places_of_part(a, part_of(a, t, kCommon, i), kCommon, false);
  most = wave_max(most);
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    upto[k] = wave_prefix_sum(places[k]);
    if (lane == 63) sums[k][wave] = upto[k];
  }
  if (lane == 0) longest[wave] = most;
  __syncthreads();
  const bool whole = a.waves && max(max(longest[0], longest[1]), max(longest[2], longest[3])) <= kWholeLen;
  int32_t at[2] = {upto[2] - places[2], whole ? upto[1] - places[1] : upto[0] - places[0]}, total[2] = {};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int32_t common = sums[2][w], mine = whole ? sums[1][w] : sums[0][w];
    at[0] += w < wave ? common : 0;
    at[1] += w < wave ? mine : 0;
    total[0] += common;
    total[1] += mine;
  }
  if (is_group) t.before_common[i] = at[0];
  if (is_seq) t.before_own[i] = at[1];
  if (i == 0) {
    t.before_common[a.n_groups] = total[0];
    t.before_common[a.n_groups + 1] = 0;
    t.before_own[a.s.n_seqs] = total[1];
    t.before_own[a.s.n_seqs + 1] = whole;
  }
  __syncthreads();
  if (blockIdx.x == 0 && i == 0) a.tables.before_own[a.s.n_seqs] = total[1];
  return t;
}

// The last of v[0 .. n - 1], which do not fall, that is at most x (v[0] is); a wave looks at 64 at a time.
template <class At>
__device__ inline int last_up_to(int n, int x, At at) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) / 64, i = lo + lane * step;
    const bool below = i < lo + n && at(i) <= x;
    const int k = max((int)__popcll(__ballot(below)) - 1, 0), next = lo + k * step;
    n = min(step, lo + n - next);
    lo = next;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// A block's or a wave's share of a line, item by item.
struct Work {
  Tables t;
  int32_t me, at, end, base, item0;
  int kind, index;
  bool undivided;                      // all items are in one piece
  Part part;
  // the piece at hand
  int head, row_block, t0, t1, tiles, all_rows;
  bool whole;
  __device__ Work(const SharedArgs& a, const Tables& t, int kind, int me) : t(t), me(me), kind(kind) {
    const Shares shares = shares_of(a, t, kind);
    undivided = shares.whole;
    at = end = 0;
    if (me >= shares.even.n) return;
    at = shares.even.begin(me);
    end = shares.even.begin(me + 1);
    index = last_up_to(a.count(kind), at, [&](int i) { return t.before(kind)[i]; });
    take(a);
  }
  __device__ void take(const SharedArgs& a) {
    const Part p = part_of(a, t, kind, index);
    auto uniform = [](int32_t x) { return __builtin_amdgcn_readfirstlane(x); };          // (scalar registers)
    part = {uniform(p.row0), uniform(p.rows), uniform(p.seq), uniform(p.page0), uniform(p.len), uniform(p.first_seen), p.each, uniform(p.common)};
    base = uniform(t.before(kind)[index]);
  }
  // Rows of the piece at hand that begins its item: the join learns where their pieces lie.  `i` of `step` lanes.
  __device__ void note_pieces(const SharedArgs& a, int i, int step) const {
    if (t0 > 0) return;
    const int row0 = row_block << a.log_rows[kind], rows = min(1 << a.log_rows[kind], all_rows - row0), n = whole ? 1 : shares_of(a, t, kind).even.owner(item0 + kItemLead + tiles - 1) - me + 1;
    for (int lr = i; lr < rows; lr += step) {
      const int64_t row = whole_row(a, row0 + lr);
      a.pieces[kind][row] = {me, n, lr, part.common};
    }
  }
  __device__ bool next(const SharedArgs& a) {
    while (at < end) {
      while (at >= base + places_of_part(a, part, kind, undivided)) {
        ++index;
        take(a);
      }
      tiles = tiles_of(part.len);
      all_rows = part.rows * a.group;
      const int row_blocks = row_blocks_of(a, part, kind), places = places_of_item(part, undivided), item = undivided ? at - base : __builtin_amdgcn_readfirstlane((uint32_t)(at - base) / (uint32_t)places),
                from = at - base - item * places;
      const Piece piece = undivided ? piece_of<kWhole>(tiles, from, end - at) : piece_of<kItemLead>(tiles, from, end - at);
      head = row_blocks == 1 ? item : __builtin_amdgcn_readfirstlane((uint32_t)item / (uint32_t)row_blocks);
      row_block = item - head * row_blocks;
      t0 = piece.first;
      t1 = piece.last;
      whole = t0 == 0 && t1 == tiles;
      item0 = at - from;
      at += piece.places;
      if (t0 < t1) return true;                            // (else the item's lead alone)
    }
    return false;
  }
  __device__ const int32_t* table(const SharedArgs& a) const { return a.s.pages + (int64_t)part.seq * a.s.max_pages + part.page0; }
  __device__ float* slot(const SharedArgs& a, int floats) const { return a.slots[kind] + (int64_t)(2 * me + (t0 == 0 ? 1 : 0)) * floats; }
  // last token that row `row` of the part (token and query head of the group) sees
  __device__ int sees(int tok) const { return part.first_seen + part.each * tok; }
  __device__ int64_t whole_row(const SharedArgs& a, int row) const { return (int64_t)(part.row0 + row / a.group) * a.hq + head * a.group + row % a.group; }
};

// The rows of the piece at hand over its tiles t0 + first, t0 + first + step, ...
// (Matrix rows behind the last have the queries of the head's first row, and nobody reads their sums.  Zeros instead would be waited for where the queries are asked for: 16 prompts of 8 beams over
// up to 8000 tokens 50.5 us, 51.7 so.)
template <int D, int Fmt, int NB>
__device__ inline void walk_piece(const SharedArgs& a, const Work& w, int lane, int first, int step, RowState<D> (&r)[NB], int& rows, int32_t* first_nan) {
  constexpr int kRows = 16 * NB;
  const int n = lane & 15, g = lane >> 4;
  int last[NB], first_seen = INT32_MAX;
  bf16x8 q[NB][D / 32];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int my_row = w.row_block * kRows + 16 * b + n;
    const bool live = my_row < w.all_rows;
    const int my_tok = live ? my_row / a.group : 0;
    last[b] = live ? w.sees(my_tok) : -1;
    first_seen = min(first_seen, live ? last[b] : INT32_MAX);
    const __bf16* x = a.q + (int64_t)(w.part.row0 + my_tok) * a.q_row + (w.head * a.group + (live ? my_row % a.group : 0)) * D + 16 * g;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) q[b][j] = *reinterpret_cast<const bf16x8*>(x + 64 * (j / 2) + 8 * (j % 2));
    r[b].m = kLow;
    r[b].l = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) r[b].o[i] = f32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int d = 8; d > 0; d >>= 1) first_seen = min(first_seen, __shfl_xor(first_seen, d));
  rows = min(w.all_rows - w.row_block * kRows, kRows);
  const int seen = w.sees((w.row_block * kRows + rows - 1) / a.group);
  const int t_end = min(w.t1, seen < 0 ? 0 : seen / kTile + 1);
  walk<D, Fmt, false>(a.c, a.scale, w.table(a), w.head, w.part.len, w.t0 + first, t_end, step, q, last, first_seen, r, nullptr, rows, nullptr, first_nan);
}

template <int D, int Fmt, int NB>
__device__ inline void few_rows(const SharedArgs& a, const Tables& t, int kind, int lane, int wave, float* stage, int32_t* first_nan) {
  constexpr int kRows = 16 * NB, kStride = D + 4;          // floats of a staged row: rows on different banks
  float* const stage_m = stage + kWaves * kRows * kStride;
  float* const stage_l = stage_m + kWaves * kRows;
  const int n = lane & 15, g = lane >> 4;
  Work w(a, t, kind, share_of_block(a, kind));
  while (w.next(a)) {
    w.note_pieces(a, threadIdx.x, 256);
    RowState<D> r[NB];
    int rows;
    walk_piece<D, Fmt, NB>(a, w, lane, wave, kWaves, r, rows, first_nan);
    float* const slot = w.slot(a, slot_floats(D, kRows));
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int lr = 16 * b + n;
      r[b].l = sum_over_groups(r[b].l);
      if (g == 0) { stage_m[wave * kRows + lr] = r[b].m; stage_l[wave * kRows + lr] = r[b].l; }
#pragma unroll
      for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(&stage[(wave * kRows + lr) * kStride + 16 * i + 4 * g]) = r[b].o[i];
    }
    __syncthreads();
    for (int j = threadIdx.x; j < rows * (D / 4); j += 256) {
      const int lr = j / (D / 4), ch = 4 * (j % (D / 4));
      float m = kLow, l = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) m = fmaxf(m, stage_m[i * kRows + lr]);
      f32x4 o = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float f = __builtin_amdgcn_exp2f(stage_m[i * kRows + lr] - m);
        l += f * stage_l[i * kRows + lr];
        o += f * *reinterpret_cast<const f32x4*>(&stage[(i * kRows + lr) * kStride + ch]);
      }
      if (w.whole) {
        float* const to = a.whole[kind] + w.whole_row(a, w.row_block * kRows + lr) * (D + 4);
        *reinterpret_cast<f32x4*>(to + ch) = o;
        if (ch == 0) { to[D] = m; to[D + 1] = l; }
      } else {
        *reinterpret_cast<f32x4*>(slot + lr * D + ch) = o;
        if (ch == 0) { slot[kRows * D + lr] = m; slot[kRows * (D + 1) + lr] = l; }
      }
    }
    __syncthreads();
  }
}

// Own parts of few rows: a wave works an item, or a piece of one, alone.  They are short as a rule - what was added behind the common beginning - and a block's waves would each have a tile or
// none, and meet for it.
template <int D, int Fmt>
__device__ inline void own_rows(const SharedArgs& a, const Tables& t, int lane, int wave, int32_t* first_nan) {
  const int n = lane & 15, g = lane >> 4;
  Work w(a, t, kOwn, kWaves * blockIdx.x + wave);
  while (w.next(a)) {
    w.note_pieces(a, lane, 64);
    RowState<D> r[1];
    int rows;
    walk_piece<D, Fmt, 1>(a, w, lane, 0, 1, r, rows, first_nan);
    r[0].l = sum_over_groups(r[0].l);
    if (n < rows) {
      float* const to = w.whole ? a.whole[kOwn] + w.whole_row(a, 16 * w.row_block + n) * (D + 4) : w.slot(a, slot_floats(D, 16)) + n * D;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(to + 16 * i + 4 * g) = r[0].o[i];
      if (g == 0) {
        float* const m = w.whole ? to + D : w.slot(a, slot_floats(D, 16)) + 16 * D + n;
        m[0] = r[0].m;
        m[w.whole ? 1 : 16] = r[0].l;
      }
    }
  }
}

template <int D, int Fmt, int kNB, bool Rest>
__device__ inline void many_rows(const SharedArgs& a, const Tables& t, int kind, int lane, int wave, unsigned char* lds, float (&key_scale)[4][4], int32_t (&live)[4][4], int32_t (&first_nan)[2][D]) {
  constexpr int kRows = 64 * kNB;
  const int n = lane & 15, g = lane >> 4;
  const RowsLane at_lane = rows_lane<D>(lane, wave);
  if (Fmt == kE4m3 && threadIdx.x < D) first_nan[1][threadIdx.x] = INT32_MAX;
  int parity = 1;                                          // of the items that see a tile
  Work w(a, t, kind, share_of_block(a, kind));
  while (w.next(a)) {
    w.note_pieces(a, threadIdx.x, 256);
    bf16x8 q[kNB][D / 32];
    f32x4 o[kNB][D / 16];
    float m[kNB], l[kNB];
    int last[kNB];
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      const int row = w.row_block * kRows + (wave * kNB + b) * 16 + n;
      const bool there = row < w.all_rows;
      const int tok = there ? row / a.group : 0;
      last[b] = there ? w.sees(tok) : -1;
      const __bf16* x = a.q + (int64_t)(w.part.row0 + tok) * a.q_row + (w.head * a.group + (there ? row % a.group : 0)) * D + 8 * g;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) q[b][j] = *reinterpret_cast<const bf16x8*>(x + 32 * j);
      m[b] = kLow;
      l[b] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) o[b][i] = f32x4{0, 0, 0, 0};
    }
    const int rows = min(w.all_rows - w.row_block * kRows, kRows), all_see = w.sees(w.row_block * kRows / a.group), seen = w.sees((w.row_block * kRows + rows - 1) / a.group);
    const int t_end = min(w.t1, seen < 0 ? 0 : seen / kTile + 1);
    if (w.t0 < t_end) {
      walk_rows<D, Fmt, kNB, Rest>(a.c, a.scale, w.table(a), w.head, w.part.len, w.t0, t_end, q, last, all_see, o, m, l, lane, wave, at_lane, lds, key_scale, live, first_nan, parity);
      parity ^= 1;
    }
#pragma unroll
    for (int b = 0; b < kNB; ++b) l[b] = sum_over_groups(l[b]);
    float* const slot = w.slot(a, slot_floats(D, kRows));
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      const int lr = (wave * kNB + b) * 16 + n, row = w.row_block * kRows + lr;
      if (!w.whole) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(slot + lr * D + 16 * i + 4 * g) = o[b][i];
        if (g == 0) { slot[kRows * D + lr] = m[b]; slot[kRows * (D + 1) + lr] = l[b]; }
      } else if (row < w.all_rows) {
        float* const to = a.whole[kind] + w.whole_row(a, row) * (D + 4);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(to + 16 * i + 4 * g) = o[b][i];
        if (g == 0) { to[D] = m[b]; to[D + 1] = l[b]; }
      }
    }
  }
}

// One launch works both lines (Own), or the line `kind`.  kRows: 16, 32, 64, 128 rows of an item.  Rest: of 64 and 128 (others always): probabilities in two parts.
template <int D, int Fmt, int kRows, bool Own, bool Rest>
__global__ __launch_bounds__(256, 2) void shared_kernel(SharedArgs a, int kind) {
  __shared__ LocalTables local;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Tables t = tables_of(a, local);
  if constexpr (kRows <= 32) {
    __shared__ __align__(16) float stage[kWaves * kRows * (D + 6)];
    __shared__ int32_t first_nan[kWaves][Fmt == kE4m3 ? D : 1];
    if constexpr (Own) own_rows<D, Fmt>(a, t, lane, wave, first_nan[wave]);
    few_rows<D, Fmt, kRows / 16>(a, t, kind, lane, wave, stage, first_nan[wave]);
  } else {
    extern __shared__ __align__(256) unsigned char lds[];  // two stages
    __shared__ float key_scale[4][4];
    __shared__ int32_t live[4][4], first_nan[2][D];
    // (the waves' own notes lie where the stages will)
    if constexpr (Own) {
      own_rows<D, Fmt>(a, t, lane, wave, reinterpret_cast<int32_t*>(lds) + wave * D);
      __syncthreads();
    }
    many_rows<D, Fmt, kRows / 64, Rest>(a, t, kind, lane, wave, lds, key_scale, live, first_nan);
  }
}

// A wave for each row: the pieces of its items.  Lane i looks at the maximum and the sum of piece i, so that all of these are asked for at once; the sums of eight pieces are on their way beside them, then of eight more.
template <int D>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedArgs a) {
  constexpr int kCh = D / 64, kAtOnce = 8;
  const int unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (unit >= a.s.n_rows * a.hq) return;
  const int tok = unit / a.hq, h = unit - tok * a.hq;
  // (all asked for at once)
  RowPieces common = a.pieces[kCommon][unit];
  const RowPieces own = a.pieces[kOwn][unit];
  const int32_t places = a.tables.before_own[a.s.n_seqs], from_row = a.s.cu[0], to_row = a.s.cu[a.s.n_seqs];
  if (places == 0 || tok < from_row || tok >= to_row) return;
  if (!own.common) common.n = 0;
  // an own part in one piece, as most are, is asked for with the stats of the others
  const bool one = __builtin_amdgcn_readfirstlane(own.n) == 1;
  const int all = __builtin_amdgcn_readfirstlane(common.n + (one ? 0 : own.n)), ch = kCh * lane;
  float m = kLow, l = 0.f, o[kCh] = {};
  if (one) {
    const float* const from = a.whole[kOwn] + (int64_t)unit * (D + 4);
    m = from[D];
    l = from[D + 1];
#pragma unroll
    for (int c = 0; c < kCh; ++c) o[c] = from[ch + c];
  }
  for (int p0 = 0; p0 < all; p0 += 64) {
    const int mine = min(p0 + lane, all - 1);
    const bool is_common = mine < common.n;
    const RowPieces x = is_common ? common : own;
    const int piece = is_common ? mine : mine - common.n, rows = 1 << (is_common ? a.log_rows[kCommon] : a.log_rows[kOwn]);
    const float* const slot = (is_common ? a.slots[kCommon] : a.slots[kOwn]) + (int64_t)(2 * (x.first + piece) + (piece == 0 ? 1 : 0)) * slot_floats(D, rows);
    const float* const whole = (is_common ? a.whole[kCommon] : a.whole[kOwn]) + (int64_t)unit * (D + 4);
    const float* const sums = x.n == 1 ? whole : slot + x.lr * D;
    const float* const stats = x.n == 1 ? whole + D : slot + rows * D + x.lr;
    const float pm = stats[0], pl = stats[x.n == 1 ? 1 : rows];
    const int n = min(all - p0, 64);
    const uint64_t at = (uint64_t)sums;
    float po[kAtOnce][kCh], next[kAtOnce][kCh];
    auto ask = [&](int j0, float (&to)[kAtOnce][kCh]) {
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int k = min(j0 + j, n - 1);
        const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)at, k), hi = __builtin_amdgcn_readlane((int)(at >> 32), k);
        const float* const from = reinterpret_cast<const float*>((uint64_t)hi << 32 | lo);
#pragma unroll
        for (int c = 0; c < kCh; ++c) to[j][c] = from[ch + c];
      }
    };
    ask(0, po);
    const float top = fmaxf(m, wave_maxf(pm)), before = __builtin_amdgcn_exp2f(m - top);
    const float f = p0 + lane < all ? __builtin_amdgcn_exp2f(pm - top) : 0.f;
    m = top;
    float part = p0 + lane < all ? f * pl : 0.f;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) part += __shfl_xor(part, d);
    l = l * before + part;
#pragma unroll
    for (int c = 0; c < kCh; ++c) o[c] *= before;
    for (int j0 = 0; j0 < n; j0 += kAtOnce) {
      if (j0 + kAtOnce < n) ask(j0 + kAtOnce, next);
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const float pf = j0 + j < n ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), min(j0 + j, n - 1))) : 0.f;
#pragma unroll
        for (int c = 0; c < kCh; ++c) {
          o[c] += j0 + j < n ? pf * po[j][c] : 0.f;
          po[j][c] = next[j][c];
        }
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  __bf16* const to = a.o + ((int64_t)tok * a.hq + h) * D + ch;
#pragma unroll
  for (int c = 0; c < kCh; ++c) to[c] = (__bf16)(o[c] * inv);
  if (lane == 0) a.lse[(int64_t)h * a.s.n_rows + tok] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---- host ---------------------------------------------------------------------------------------

// Rows of a block, from the rows of a group or a sequence on average (as in fcp_cache_attn).
int rows_form(int64_t all_rows, int64_t n) { return all_rows <= 16 * n ? 16 : all_rows <= 32 * n ? 32 : all_rows <= 64 * n ? 64 : 128; }

struct SharedPlan { int rows[2]; int32_t sharers[2]; bool waves, local; };
SharedPlan plan_shared(const CacheView& c, int32_t n_seqs, int32_t n_groups, int32_t tq, int32_t hq) {
  SharedPlan p;
  const int64_t all_rows = (int64_t)tq * (hq / c.hkv);
  p.rows[kCommon] = rows_form(all_rows, n_groups);
  p.rows[kOwn] = rows_form(all_rows, n_seqs);
  p.waves = p.rows[kOwn] == 16;
  p.sharers[kCommon] = kBlocks;
  p.sharers[kOwn] = p.waves ? kSharers : kBlocks;
  p.local = n_seqs <= kLocal;
  return p;
}
// Scratch: for any number of groups up to n_seqs.  The slots of common parts have room for the rows of one group.
struct SharedSpace { size_t parts[2], before[2], pieces[2], slots[2], whole[2], bytes; };
// Whether every sequence is worked by itself, as fcp_cache_attn does.  Many rows of a sequence are attention of many rows already: the matrix units bound it, and the bytes that sequences share are read from
// the L2s (8 questions of 256 tokens about 4000: 221 us so, 328 in groups).  Else what groups gain is bytes, and what they cost is the second part and its joining, 8 to 15 us of a call, more with two
// launches.  How long the common parts are only the device knows; what they may save at most follows from the tables' size.  Itself / in groups, e4m3, 32 query heads over 8 KV heads, MB that may be saved:
// 4 rows for a KV head 4 MB 8 / 18 us, 63 19.8 / 19.4, 73 20 / 26, 135 28 / 30, 251 43 / 30 and 33 / 27, 500 58 / 36, 2200 174 / 64; 8 rows 251 MB 46 / 36 and 34 / 36, 520 54 / 46; 16 rows 123 MB 29 / 36, 503 80 / 57 and
// 54 / 65, 1000 92 / 79, 2200 188 / 144; 64 rows 63 MB 37 / 55, 478 134 / 119, 2200 456 / 338.  17 to 32 rows gain little or nothing, since both ways multiply probabilities in two parts and the products are
// what bounds them: 32 rows 123 MB 39 / 55, 478 92 / 92, 985 118 / 144, 2200 230 / 242.
bool by_itself(const CacheView& c, int head_dim, int32_t n_seqs, int32_t n_groups, int32_t max_pages, int32_t tq, int32_t hq) {
  const int64_t rows = (int64_t)tq * (hq / c.hkv), saved = n_groups == 0 ? 0 : (int64_t)(n_seqs - n_groups) * max_pages * c.page * c.hkv * 2 * head_dim;
  return rows > (int64_t)64 * n_seqs || saved < (int64_t)(rows <= (int64_t)8 * n_seqs ? 1 : 3) << 27;
}
SharedSpace shared_space(const CacheView& c, int head_dim, int32_t n_seqs, int32_t tq, int32_t hq) {
  SharedSpace s;
  const SharedPlan p = plan_shared(c, n_seqs, 1, tq, hq);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += pad_to(bytes, 256); return here; };
  for (int kind = 0; kind < 2; ++kind) {
    s.parts[kind] = take((size_t)n_seqs * sizeof(Entry));
    s.before[kind] = take(((size_t)n_seqs + 2) * 4);
    s.pieces[kind] = take((size_t)tq * hq * sizeof(RowPieces));
    s.slots[kind] = take((size_t)2 * p.sharers[kind] * slot_floats(head_dim, p.rows[kind]) * 4);
    s.whole[kind] = take((size_t)tq * hq * (head_dim + 4) * 4);
  }
  s.bytes = at;
  return s;
}

template <int D, int Fmt, int kRows, bool Own, bool Rest>
int launch_line(const SharedArgs& a, int kind, hipStream_t st) {
  constexpr int kLds = kRows <= 32 ? 0 : 2 * Stage<D>::kBytes;
  auto kernel = shared_kernel<D, Fmt, kRows, Own, Rest>;
  if (kLds > 48 * 1024) {
    static std::atomic<uint64_t> raised;
    if (int rc = raise_lds_limit(reinterpret_cast<const void*>(kernel), kLds, raised)) return rc;
  }
  kernel<<<dim3((unsigned)kBlocks), dim3(256), kLds, st>>>(a, kind);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}

template <int D, int Fmt>
int launch_shared(const SharedArgs& a, hipStream_t st) {
  if (!a.local) {
    parts_kernel<<<dim3(1), dim3(kPartThreads), 0, st>>>(a);
    FCP_HIP_CHECK(hipGetLastError());
  }
  const int common = 1 << a.log_rows[kCommon];
  int rc;
  // Probabilities are as exact as fcp_cache_attn has them for the same sequences: in two parts, however many rows a group brings together, but where sequences have more than 32 rows.
  if (a.waves) {
    rc = common == 16 ? launch_line<D, Fmt, 16, true, true>(a, kCommon, st) : common == 32 ? launch_line<D, Fmt, 32, true, true>(a, kCommon, st)
       : common == 64 ? launch_line<D, Fmt, 64, true, true>(a, kCommon, st) : launch_line<D, Fmt, 128, true, true>(a, kCommon, st);
  } else if (a.log_rows[kOwn] == 5) {
    rc = common == 32 ? launch_line<D, Fmt, 32, false, true>(a, kCommon, st) : common == 64 ? launch_line<D, Fmt, 64, false, true>(a, kCommon, st)
       : launch_line<D, Fmt, 128, false, true>(a, kCommon, st);
    if (!rc) rc = launch_line<D, Fmt, 32, false, true>(a, kOwn, st);
  } else {
    rc = common == 64 ? launch_line<D, Fmt, 64, false, false>(a, kCommon, st) : launch_line<D, Fmt, 128, false, false>(a, kCommon, st);
    if (!rc) rc = launch_line<D, Fmt, 64, false, false>(a, kOwn, st);
  }
  if (rc) return rc;
  shared_join_kernel<D><<<dim3((unsigned)(((int64_t)a.s.n_rows * a.hq + 3) / 4)), dim3(256), 0, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}

int check_shared(const char* who, const CacheView& c, int32_t n_seqs, int32_t max_pages, int32_t tq, int32_t hq) {
  if (int rc = check_heads(who, c, hq)) return rc;
  if (int rc = check_row_count(who, tq, hq)) return rc;
  // (most places: with as many groups as sequences, rows in blocks of 16)
  const int64_t tiles = max(((int64_t)max_pages * c.page + kTile - 1) / kTile, (int64_t)1);
  if ((tiles + kItemLead) * c.hkv * (n_seqs + (int64_t)tq * (hq / c.hkv) / 16) > kMostPlaces || !fits_axis(((int64_t)tq * hq + 3) / 4, 256))
    return fail(FCP_ERR_UNSUPPORTED, "%s: tables and rows that may make 2^31 tiles of work", who);
  return FCP_OK;
}

}  // namespace

// 0: refused
size_t shared_scratch_bytes(const char* who, const CacheView& c, int head_dim, int32_t n_seqs, int32_t max_pages, int32_t tq, int32_t hq) {
  if (check_shared(who, c, n_seqs, max_pages, tq, hq)) return 0;
  const size_t itself = attn_scratch_bytes(c, head_dim, n_seqs, max_pages, tq, hq);
  if (by_itself(c, head_dim, n_seqs, 1, max_pages, tq, hq)) return itself;
  return max(itself, shared_space(c, head_dim, n_seqs, tq, hq).bytes);         // (with more groups less may be saved)
}

}  // namespace fcp

extern "C" int fcp_cache_attn_shared(const fcp_cache* cache, const void* q, int64_t q_row, int32_t tq, int32_t hq, const int32_t* cu_seqlens, const int32_t* kv_len,
                                     const int32_t* pages, int32_t n_seqs, int32_t max_pages, const int32_t* groups, const int32_t* shared_len, int32_t n_groups,
                                     float softmax_scale, void* o, float* lse, void* scratch, size_t scratch_bytes, void* stream) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_cache_attn_shared";
  SharedArgs a = {};
  if (int rc = check_cache(who, cache, false, &a.c)) return rc;
  if (int rc = check_heads(who, a.c, hq)) return rc;
  if (int rc = check_seqs(who, a.c, cu_seqlens, true, kv_len, pages, n_seqs, max_pages, tq)) return rc;
  if (int rc = check_scale(who, softmax_scale)) return rc;
  if (n_groups < 0 || n_groups > n_seqs || (n_groups > 0 && (!groups || !shared_len)))
    return fail(FCP_ERR_INVALID_ARG, "%s: %d groups of %d sequences need their first sequences and lengths", who, n_groups, n_seqs);
  if (int rc = check_int_pointers(who, {groups, shared_len})) return rc;
  if (tq == 0 || n_seqs == 0) return FCP_OK;
  if (int rc = check_rows(who, cache, q, q_row, tq, hq)) return rc;
  if (!o || !lse || (uintptr_t)o % 16 || (uintptr_t)lse % 4) return fail(FCP_ERR_INVALID_ARG, "%s: o and lse are required and must be aligned", who);
  if (!scratch || (uintptr_t)scratch % 256) return fail(FCP_ERR_INVALID_ARG, "%s: scratch must be 256-byte aligned", who);
  if (int rc = check_shared(who, a.c, n_seqs, max_pages, tq, hq)) return rc;
  const size_t need = shared_scratch_bytes(who, a.c, cache->head_dim, n_seqs, max_pages, tq, hq);
  if (scratch_bytes < need) return fail(FCP_ERR_CAPACITY, "%s: scratch has %zu bytes, %zu are needed", who, scratch_bytes, need);
  if (by_itself(a.c, cache->head_dim, n_seqs, n_groups, max_pages, tq, hq))
    return fcp_cache_attn(cache, q, q_row, tq, hq, cu_seqlens, kv_len, pages, n_seqs, max_pages, softmax_scale, 0, o, lse, scratch, scratch_bytes, stream);
  const SharedSpace space = shared_space(a.c, cache->head_dim, n_seqs, tq, hq);
  const SharedPlan p = plan_shared(a.c, n_seqs, n_groups, tq, hq);
  a.s = {cu_seqlens, kv_len, pages, n_seqs, max_pages, tq};
  a.groups = groups;
  a.shared_len = shared_len;
  a.n_groups = n_groups;
  a.q = static_cast<const __bf16*>(q);
  a.q_row = q_row;
  a.hq = hq;
  a.group = hq / a.c.hkv;
  a.scale = softmax_scale * kLog2e;
  a.o = static_cast<__bf16*>(o);
  a.lse = lse;
  char* const at = static_cast<char*>(scratch);
  a.tables = {reinterpret_cast<Entry*>(at + space.parts[kCommon]), reinterpret_cast<Entry*>(at + space.parts[kOwn]), reinterpret_cast<int32_t*>(at + space.before[kCommon]),
              reinterpret_cast<int32_t*>(at + space.before[kOwn])};
  for (int kind = 0; kind < 2; ++kind) {
    a.pieces[kind] = reinterpret_cast<RowPieces*>(at + space.pieces[kind]);
    a.slots[kind] = reinterpret_cast<float*>(at + space.slots[kind]);
    a.whole[kind] = reinterpret_cast<float*>(at + space.whole[kind]);
    a.log_rows[kind] = __builtin_ctz(p.rows[kind]);
    a.log_sharers[kind] = __builtin_ctz(p.sharers[kind]);
  }
  a.waves = p.waves;
  a.local = p.local;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool e4m3 = cache->format == FCP_CACHE_E4M3;
  return cache->head_dim == 128 ? (e4m3 ? launch_shared<128, kE4m3>(a, st) : launch_shared<128, kInt8>(a, st))
                                : (e4m3 ? launch_shared<64, kE4m3>(a, st) : launch_shared<64, kInt8>(a, st));
}
