// fcp_cache_fork and fcp_cache_compact: who holds which page of the cache, kept on the device.
//
// A sequence that continues another one takes over its table; pages that are only read are shared, and a page that new tokens go into is copied for all of those who would write it but one.
// Every entry of this step's tables is looked at once, and marks its page; then one block counts through the marks for free pages, in increasing order, and lists the copies; the last launch copies,
// 16 bytes a thread, a block for each (page, KV head), whose keys are one run of memory and whose values are another, and writes the tables.
// Small calls are chains of loads and launches.  Where the tables are not large the block that plans marks too, bits in LDS: two launches; else four, with a byte a page.
//
// A step of 8 beams 11.0 us, of 32 prompts' 256 over up to 8001 tokens 14.4 (planning 7 and 10 of them); 1024 beams that begin, of 64 prompts, 38 (planning 16, copying 19: 136 MB read and
// written); 8 sequences compacted 12.3, 64 of up to 16384 tokens 145 (planning 14, copying 129: 635 MB read and written, a copy's rate).
#include "fcp_cache.h"

namespace fcp {
namespace {

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;

struct Copy { int32_t from, to, tokens, copied; };         // copied: fork, the entry is a copy's, whether there was a page for it or not

struct PageArgs {
  CacheView c;
  SeqView s;                           // this step's sequences (no rows); rows of both tables are max_pages long
  const int32_t* parent;               // fork: [n_new]
  const int32_t* news;
  int32_t n_new;
  const uint8_t* busy;
  int32_t* new_pages;
  int32_t* new_len;
  int32_t* counts;
  // scratch
  uint8_t* held;                       // large calls, a byte a page: sequences of this step (fork: or others) hold it
  uint8_t* read;                       // fork: sequences of the next step (or others) hold it and do not write it
  int32_t* lowest;                     // fork: of the sequences of the next step that would write a page, the lowest; compact: where a page moves.  Only entries of such pages mean something
  int32_t* list;                       // fork: free pages; compact: pages in which others move
  Copy* copies;
  int32_t* n_copies;                   // compact: pages that move, and the first number past those in use afterwards
  int32_t words;                       // of a bit a page
};

__device__ inline int32_t cached(const PageArgs& a, int seq) {
  const int64_t room = (int64_t)a.s.max_pages << a.c.log_page;
  const int32_t n = max(a.s.kv_len[seq], 0);
  return n < room ? n : (int32_t)room;
}
// A sequence of the next step: whom it continues (-1: nobody), tokens before and after, the place of the page in which both lie (-1: there is none).
struct Next { int32_t parent, before, after, writes; };
__device__ inline Next next_of(const PageArgs& a, int seq) {
  const int32_t p = a.parent[seq], n = max(a.news[seq], 0);
  const bool there = (uint32_t)p < (uint32_t)a.s.n_seqs;
  const int32_t before = there ? cached(a, p) : 0;
  const int64_t after = min((int64_t)before + n, (int64_t)a.s.max_pages << a.c.log_page);
  return {there ? p : -1, before, (int32_t)after, after > before && (before & (a.c.page - 1)) ? before >> a.c.log_page : -1};
}
__device__ inline int32_t pages_for(const PageArgs& a, int32_t tokens) { return (int32_t)(((int64_t)tokens + a.c.page - 1) >> a.c.log_page); }
__device__ inline int32_t entry(const PageArgs& a, int seq, int place) {
  const int32_t p = a.s.pages[(int64_t)seq * a.s.max_pages + place];
  return (uint32_t)p < (uint32_t)a.c.n_pages ? p : -1;
}
// Sum over the block before this thread, and of all threads.  Every thread calls.
struct Scan { int32_t before, all; };
__device__ inline Scan block_scan(int32_t x, int32_t* sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // (two counts in a word may reach its sign)
  const uint32_t upto = wave_prefix(x, [](int32_t a, int32_t b) { return (int32_t)((uint32_t)a + (uint32_t)b); });
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  uint32_t before = upto - (uint32_t)x, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const uint32_t n = sums[w];
    before += w < wave ? n : 0;
    all += n;
  }
  __syncthreads();
  return {(int32_t)before, (int32_t)all};
}

// Two counts of up to 33 a thread, in the halves of a word: the block's are below 2^16.
struct Pair { Scan low, high; };
__device__ inline Pair pair_of(const Scan& x) {
  return {{x.before & 0xffff, x.all & 0xffff}, {(int32_t)((uint32_t)x.before >> 16), (int32_t)((uint32_t)x.all >> 16)}};
}

// A word of bits, one for each of 32 bytes that is not 0 (behind n: 0).
__device__ inline uint32_t bits_of(const uint8_t* bytes, int w, int32_t n) {
  uint32_t bits = 0;
  if (!bytes) return 0;
  if (32 * w + 32 <= n) {
    struct __attribute__((packed, aligned(1))) Words { uint32_t x[8]; };
    const Words r = *reinterpret_cast<const Words*>(bytes + 32 * (int64_t)w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t x = r.x[i];
      x |= x >> 4;
      x |= x >> 2;
      x = (x | x >> 1) & 0x01010101u;
      bits |= (x * 0x01020408u >> 24) << 4 * i;            // (the bytes' bits next to each other, the first one lowest)
    }
  } else {
    for (int i = 32 * w; i < n; ++i) bits |= (uint32_t)(bytes[i] != 0) << (i - 32 * w);
  }
  return bits;
}

// The marks of pages, as bits in LDS or as bytes in scratch.
// In LDS two bits a page, 16 pages a word: held, read (compact: busy), so that an entry is marked with one addition of bits.
__device__ inline uint32_t even_bits(uint32_t x) {         // bits 0, 2, 4, .. next to each other
  x &= 0x55555555u;
  x = (x | x >> 1) & 0x33333333u;
  x = (x | x >> 2) & 0x0f0f0f0fu;
  x = (x | x >> 4) & 0x00ff00ffu;
  return (x | x >> 8) & 0xffffu;
}
__device__ inline uint32_t spread_bits(uint32_t x) {       // 16 bits to bits 0, 2, 4, ..
  x &= 0xffffu;
  x = (x | x << 8) & 0x00ff00ffu;
  x = (x | x << 4) & 0x0f0f0f0fu;
  x = (x | x << 2) & 0x33333333u;
  return (x | x << 1) & 0x55555555u;
}
constexpr uint32_t kHeld = 1, kRead = 2;
struct LdsMarks {
  uint32_t* two;
  __device__ uint32_t held_word(int w) const { return even_bits(two[2 * w]) | even_bits(two[2 * w + 1]) << 16; }
  __device__ uint32_t read_word(int w) const { return even_bits(two[2 * w] >> 1) | even_bits(two[2 * w + 1] >> 1) << 16; }
  __device__ bool is_read(int32_t page) const { return two[page >> 4] >> 2 * (page & 15) & kRead; }
};
struct ByteMarks {
  const uint8_t* held;
  const uint8_t* read;
  int32_t n;
  __device__ uint32_t held_word(int w) const { return bits_of(held, w, n); }
  __device__ uint32_t read_word(int w) const { return bits_of(read, w, n); }
  __device__ bool is_read(int32_t page) const { return read && read[page]; }
};

// ---- large calls: marks ------------------------------------------------------------------------------------------
template <bool Fork>
__global__ __launch_bounds__(256) void clear_kernel(PageArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  for (int j = 4 * i; j < min(4 * i + 4, a.c.n_pages); ++j) {
    const uint8_t b = a.busy ? a.busy[j] : 0;
    a.held[j] = Fork ? b : 0;
    if (Fork) a.read[j] = b;
  }
  if (Fork && i < a.n_new) {
    const Next x = next_of(a, i);
    const int32_t page = x.writes >= 0 ? entry(a, x.parent, x.writes) : -1;
    if (page >= 0) a.lowest[page] = INT32_MAX;
  }
}

// All entries, a wave for 64 places of a sequence.  (Who marks a page first does not matter: the same byte is written.)
template <bool Fork>
__global__ __launch_bounds__(256) void mark_kernel(PageArgs a) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int per_seq = (a.s.max_pages + 63) / 64;
  const int64_t seq = unit / per_seq;
  const int place = (int)(unit % per_seq) * 64 + (threadIdx.x & 63);
  if (place >= a.s.max_pages) return;
  if (seq < a.s.n_seqs) {
    if (place < pages_for(a, cached(a, (int)seq))) {
      const int32_t page = entry(a, (int)seq, place);
      if (page >= 0) a.held[page] = 1;
    }
  } else if (Fork && seq - a.s.n_seqs < a.n_new) {
    const int i = (int)(seq - a.s.n_seqs);
    const Next x = next_of(a, i);
    const int32_t page = place < pages_for(a, x.before) ? entry(a, x.parent, place) : -1;
    if (page >= 0) {
      if (place == x.writes) atomicMin(a.lowest + page, i);
      else a.read[page] = 1;
    }
  }
}

// ---- small calls: the block that plans marks -----------------------------------------------------------------------
// One block / many, us, tables all but full, fork and compact: 8 sequences of 64 entries 8.8 / 13.7 and 8.5 / 12.0, 64 of 256 12.2 / 16.0 and 11.0 / 14.4, 256 of 127 14.4 / 16.1, of 256 20.1 / 14.4 and
// 16.9 / 11.8, 1024 of 128 35.4 / 17.6 and 29.0 / 12.4; 64 of 64 in a pool of 200000 pages 17.2 / 24.2 and 19.5 / 24.4.  The others are what LDS has room for, and a thread for each new sequence.
constexpr int kLdsPages = 1 << 18, kLdsSeqs = 4096, kLdsEntries = 1 << 15, kLdsNew = kPlanThreads;
// Per page: marks, and whether somebody writes it; per sequence of this step: whether it has children, whether one of them goes on without new tokens in a page that is begun, its tokens, the
// lowest child that writes its last page.
struct LdsTables { LdsMarks marks; uint32_t *written, *child, *part; int32_t *len, *low; };
__host__ __device__ inline size_t lds_bytes(int32_t words, int32_t n_seqs) { return (size_t)12 * words + 8 * ((n_seqs + 31) / 32) + 8 * (size_t)n_seqs; }
__device__ inline LdsTables lds_tables(const PageArgs& a, unsigned char* lds) {
  const int seq_words = (a.s.n_seqs + 31) / 32;
  uint32_t* const two = reinterpret_cast<uint32_t*>(lds);
  uint32_t* const child = two + 3 * a.words;
  int32_t* const len = reinterpret_cast<int32_t*>(child + 2 * seq_words);
  return {{two}, two + 2 * a.words, child, child + seq_words, len, len + a.s.n_seqs};
}
__device__ inline void set_bit(uint32_t* bits, int32_t i) { atomicOr(bits + (i >> 5), 1u << (i & 31)); }
__device__ inline bool bit(const uint32_t* bits, int32_t i) { return bits[i >> 5] >> (i & 31) & 1; }

// Clears the marks but those of busy pages, and looks up the lengths.
template <bool Fork>
__device__ inline void begin_marks(const PageArgs& a, const LdsTables& t) {
  for (int w = threadIdx.x; w < a.words; w += kPlanThreads) {
    const uint32_t b = bits_of(a.busy, w, a.c.n_pages);
#pragma unroll
    for (int half = 0; half < 2; ++half) t.marks.two[2 * w + half] = spread_bits(b >> 16 * half) * (Fork ? kHeld | kRead : kRead);
    if (Fork) t.written[w] = 0;
  }
  for (int s = threadIdx.x; s < a.s.n_seqs; s += kPlanThreads) {
    t.len[s] = cached(a, s);
    if (Fork) t.low[s] = INT32_MAX;
  }
  for (int w = threadIdx.x; w < (a.s.n_seqs + 31) / 32; w += kPlanThreads) t.child[w] = t.part[w] = 0;
}
// Marks this step's entries; fork: as read by others too, those of sequences with children, but the page in which new tokens go, which is marked if a child goes on without any.
template <bool Fork>
__device__ inline void mark_in_lds(const PageArgs& a, const LdsTables& t) {
  // Four neighbouring entries a lane, 16 to 64 lanes a sequence, as the tables are long; a wave looks at eight such lots at once, so that their loads are on the way together.  Instructions bound
  // this where there are thousands of entries for each wave, so there are few for an entry: a mark is made whether it is there or not (256 beams 14.4 us; 22.9 with a look before).
  constexpr int kAtOnce = 8;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int log_lanes = a.s.max_pages > 128 ? 6 : a.s.max_pages > 64 ? 5 : 4, of_lot = 64 >> log_lanes, sub = lane >> log_lanes;
  for (int first = 0; first < a.s.max_pages; first += 4 << log_lanes)
    for (int lot = wave; lot * of_lot < a.s.n_seqs; lot += kAtOnce * kPlanWaves) {
      const int place = first + 4 * (lane & ((1 << log_lanes) - 1));
      int32_t page[kAtOnce][4];
      int readable[kAtOnce];                               // places before this one are read by others
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int seq = (lot + k * kPlanWaves) * of_lot + sub;
        const bool there = seq < a.s.n_seqs;
        const int32_t len = there ? t.len[seq] : 0, n = pages_for(a, len);
        readable[k] = Fork && there && bit(t.child, seq) ? (bit(t.part, seq) ? n : len >> a.c.log_page) : 0;
        const int32_t* const from = a.s.pages + (int64_t)(there ? seq : 0) * a.s.max_pages + place;
        struct __attribute__((packed, aligned(4))) Four { int32_t x[4]; };
        Four f = {{-1, -1, -1, -1}};
        if (place + 4 <= n) {
          f = *reinterpret_cast<const Four*>(from);
        } else if (place < n) {
#pragma unroll
          for (int j = 0; j < 3; ++j) f.x[j] = place + j < n ? from[j] : -1;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) page[k][j] = f.x[j];
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t x = page[k][j];
          if (x < (uint32_t)a.c.n_pages) atomicOr(t.marks.two + (x >> 4), (place + j < readable[k] ? kHeld | kRead : kHeld) << (2 * x & 31));
        }
    }
}

// ---- one block hands out pages -------------------------------------------------------------------------------------
template <class Marks>
__device__ inline void plan_fork(const PageArgs& a, const Marks& marks) {
  __shared__ int32_t sums[kPlanWaves];
  auto copied = [&](int i, const Next& x, int32_t& page) {
    page = x.writes >= 0 ? entry(a, x.parent, x.writes) : -1;
    return page >= 0 && (marks.is_read(page) || __hip_atomic_load(a.lowest + page, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != i);
  };
  // pages that are needed, and those that nobody holds but who writes them
  int32_t need = 0, kept = 0;
  for (int i = threadIdx.x; i < a.n_new; i += kPlanThreads) {
    const Next x = next_of(a, i);
    int32_t page;
    const bool copy = copied(i, x, page);
    need += copy + pages_for(a, x.after) - pages_for(a, x.before);
    kept += page >= 0 && !copy;
    a.new_len[i] = x.after;
  }
  need = block_scan(need, sums).all;
  int32_t listed = 0;
  for (int w0 = 0; w0 < a.words; w0 += kPlanThreads) {
    const int w = w0 + threadIdx.x;
    uint32_t free = w < a.words ? ~marks.held_word(w) : 0u;
    if (w == a.words - 1 && a.c.n_pages % 32) free &= (1u << (a.c.n_pages % 32)) - 1;
    kept += w < a.words ? __popc(marks.read_word(w)) : 0;
    const Scan at = block_scan(__popc(free), sums);
    int32_t rank = listed + at.before;
    for (; free && rank < need; free &= free - 1) a.list[rank++] = 32 * w + __builtin_ctz(free);
    listed += at.all;
  }
  kept = block_scan(kept, sums).all;                       // (pages that the next step's sequences hold already, or others)
  const int32_t taken = min(need, listed);
  if (threadIdx.x == 0) {
    a.counts[0] = taken;
    a.counts[1] = need - taken;
    a.counts[2] = a.c.n_pages - kept - taken;
  }
  int32_t before = 0;
  for (int i0 = 0; i0 < a.n_new; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    Next x = {};
    int32_t page = -1;
    bool copy = false;
    if (i < a.n_new) {
      x = next_of(a, i);
      copy = copied(i, x, page);
    }
    const Scan at = block_scan(i < a.n_new ? copy + pages_for(a, x.after) - pages_for(a, x.before) : 0, sums);
    if (i < a.n_new) {
      int32_t rank = before + at.before;
      int32_t* const table = a.new_pages + (int64_t)i * a.s.max_pages;
      auto next = [&] { const int32_t r = rank++; return r < taken ? a.list[r] : -1; };
      Copy c = {page, -1, 0, copy};
      if (copy) {
        c.to = table[x.writes] = next();
        c.tokens = c.to >= 0 ? x.before & (a.c.page - 1) : 0;
      }
      a.copies[i] = c;
      for (int place = pages_for(a, x.before); place < pages_for(a, x.after); ++place) table[place] = next();
    }
    before += at.all;
  }
}
__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(PageArgs a) { plan_fork(a, ByteMarks{a.held, a.read, a.c.n_pages}); }

// A new sequence a thread, whose numbers stay in registers; free pages in LDS as far as they fit.  (What this takes is loads that wait for each other, 0.7 us each.)
__global__ __launch_bounds__(kPlanThreads) void fork_small_kernel(PageArgs a) {
  constexpr int kListed = 2 * kPlanThreads;
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ int32_t sums[kPlanWaves], list[kListed], written[kPlanThreads], several;           // written: pages that the sequences would write, or -1
  const LdsTables t = lds_tables(a, lds);
  const int i = threadIdx.x;
  const bool there = i < a.n_new;
  const int32_t said = there ? a.parent[i] : -1, news = there ? max(a.news[i], 0) : 0;
  begin_marks<true>(a, t);
  __syncthreads();
  const int32_t parent = (uint32_t)said < (uint32_t)a.s.n_seqs ? said : -1, tokens = parent >= 0 ? t.len[parent] : 0;
  const int32_t after = (int32_t)min((int64_t)tokens + news, (int64_t)a.s.max_pages << a.c.log_page), writes = after > tokens && (tokens & (a.c.page - 1)) ? tokens >> a.c.log_page : -1;
  const int32_t page = writes >= 0 ? entry(a, parent, writes) : -1;
  if (parent >= 0) {
    if (!bit(t.child, parent)) set_bit(t.child, parent);
    if (writes < 0 && !bit(t.part, parent)) set_bit(t.part, parent);
  }
  if (i == 0) several = 0;
  __syncthreads();
  mark_in_lds<true>(a, t);
  if (page >= 0) atomicMin(t.low + parent, i);             // (the page was asked for before the marks' entries, and is waited for with them)
  written[i] = page;
  __syncthreads();
  const bool lowest = page >= 0 && t.low[parent] == i;
  if (lowest && (atomicOr(t.written + (page >> 5), 1u << (page & 31)) >> (page & 31) & 1)) several = 1;    // two parents have begun the same page
  __syncthreads();
  // whether one before it would write the page too
  bool copy = page >= 0 && !lowest;
  if (several)
    for (int j = 0; page >= 0 && j < i; ++j) copy |= written[j] == page;
  copy |= page >= 0 && t.marks.is_read(page);
  const Scan mine = block_scan(copy + pages_for(a, after) - pages_for(a, tokens), sums);
  const int32_t need = mine.all;
  int32_t listed = 0, held = 0;
  for (int w0 = 0; w0 < a.words; w0 += kPlanThreads) {
    const int w = w0 + i;
    uint32_t free = w < a.words ? ~t.marks.held_word(w) : 0u;
    if (w == a.words - 1 && a.c.n_pages % 32) free &= (1u << (a.c.n_pages % 32)) - 1;
    const int32_t kept = (w < a.words ? __popc(t.marks.read_word(w)) : 0) + (w0 == 0 && page >= 0 && !copy);
    const Pair at = pair_of(block_scan((int32_t)(__popc(free) | (uint32_t)kept << 16), sums));
    int32_t rank = listed + at.low.before;
    for (; free && rank < need; free &= free - 1, ++rank) (rank < kListed ? list : a.list)[rank] = 32 * w + __builtin_ctz(free);
    listed += at.low.all;
    held += at.high.all;
  }
  __syncthreads();                                         // (the list is written)
  const int32_t taken = min(need, listed);
  if (i == 0) {
    a.counts[0] = taken;
    a.counts[1] = need - taken;
    a.counts[2] = a.c.n_pages - held - taken;
  }
  if (!there) return;
  int32_t rank = mine.before;
  int32_t* const table = a.new_pages + (int64_t)i * a.s.max_pages;
  auto next = [&] { const int32_t r = rank++; return r >= taken ? -1 : r < kListed ? list[r] : a.list[r]; };
  Copy c = {page, -1, 0, copy};
  if (copy) {
    c.to = table[writes] = next();
    c.tokens = c.to >= 0 ? tokens & (a.c.page - 1) : 0;
  }
  a.copies[i] = c;
  a.new_len[i] = after;
  for (int place = pages_for(a, tokens); place < pages_for(a, after); ++place) table[place] = next();
}

// The pages in use move to the lowest numbers that are not busy: `end` is the first number past these.
template <class Marks>
__device__ inline void plan_compact(const PageArgs& a, const Marks& marks) {
  __shared__ int32_t sums[kPlanWaves];
  __shared__ int32_t end_at, busy_end;
  auto busy_bits = [&](int w) { return marks.read_word(w); };
  if (threadIdx.x == 0) end_at = busy_end = 0;
  __syncthreads();
  int32_t used = 0, all = 0;
  for (int w0 = 0; w0 < a.words; w0 += kPlanThreads) {
    const int w = w0 + threadIdx.x;
    const uint32_t h = w < a.words ? marks.held_word(w) : 0u, b = w < a.words ? busy_bits(w) : 0u;
    if (b) atomicMax(&busy_end, 32 * w + 32 - __builtin_clz(b));
    const Pair n = pair_of(block_scan((int32_t)(__popc(h & ~b) | (uint32_t)__popc(h) << 16), sums));
    used += n.low.all;
    all += n.high.all;
  }
  // the used-th page that is not busy
  int32_t seen = 0;
  for (int w0 = 0; w0 < a.words && seen < used; w0 += kPlanThreads) {
    const int w = w0 + threadIdx.x;
    uint32_t open = w < a.words ? ~busy_bits(w) : 0u;
    const Scan at = block_scan(__popc(open), sums);
    int32_t rank = seen + at.before;
    if (rank < used && rank + __popc(open) >= used) {
      for (; rank + 1 < used; ++rank) open &= open - 1;
      end_at = 32 * w + __builtin_ctz(open) + 1;
    }
    seen += at.all;
  }
  __syncthreads();
  const int32_t end = end_at;
  int32_t holes = 0, movers = 0;
  for (int w0 = 0; w0 < a.words; w0 += kPlanThreads) {
    const int w = w0 + threadIdx.x;
    uint32_t hole = 0, mover = 0;
    if (w < a.words) {
      const uint32_t h = marks.held_word(w), b = busy_bits(w), low = 32 * w + 32 <= end ? ~0u : 32 * w >= end ? 0u : (1u << (end - 32 * w)) - 1;
      hole = low & ~h & ~b;
      mover = ~low & h & ~b;
    }
    const Pair n = pair_of(block_scan((int32_t)(__popc(hole) | (uint32_t)__popc(mover) << 16), sums));
    int32_t rank = holes + n.low.before;
    for (; hole; hole &= hole - 1) a.list[rank++] = 32 * w + __builtin_ctz(hole);
    rank = movers + n.high.before;
    for (; mover; mover &= mover - 1) a.copies[rank++] = {32 * w + __builtin_ctz(mover), -1, a.c.page, 0};
    holes += n.low.all;
    movers += n.high.all;
  }
  __threadfence_block();
  __syncthreads();
  for (int i = threadIdx.x; i < movers; i += kPlanThreads) {
    const int32_t from = a.copies[i].from, to = a.list[i];
    a.copies[i].to = to;
    a.lowest[from] = to;
  }
  if (threadIdx.x == 0) {
    a.counts[0] = movers;
    a.counts[1] = all;
    a.counts[2] = max(end, busy_end);
    a.n_copies[0] = movers;
    a.n_copies[1] = end;
  }
}
__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(PageArgs a) { plan_compact(a, ByteMarks{a.held, a.busy, a.c.n_pages}); }
__global__ __launch_bounds__(kPlanThreads) void compact_small_kernel(PageArgs a) {
  extern __shared__ __align__(16) unsigned char lds[];
  const LdsTables t = lds_tables(a, lds);
  begin_marks<false>(a, t);
  __syncthreads();
  mark_in_lds<false>(a, t);
  __syncthreads();
  plan_compact(a, t.marks);
}

// ---- last launch --------------------------------------------------------------------------------------------------
// The first `tokens` tokens of a (page, KV head), values in whole groups.
__device__ inline void copy_page(const CacheView& c, int head_dim, const Copy& x, int head) {
  const int64_t from = block_of(c, x.from, head), to = block_of(c, x.to, head);
  const int row = head_dim / 16, keys = x.tokens * row, values = (x.tokens + kGroup - 1) / kGroup * kGroup * row;
  const u32x4* const k0 = reinterpret_cast<const u32x4*>(c.k) + from * c.page * row;
  const u32x4* const v0 = reinterpret_cast<const u32x4*>(c.v) + from * c.page * row;
  u32x4* const k1 = reinterpret_cast<u32x4*>(c.k) + to * c.page * row;
  u32x4* const v1 = reinterpret_cast<u32x4*>(c.v) + to * c.page * row;
  for (int i = threadIdx.x; i < values; i += 256) {
    const bool key = i < keys;
    const u32x4 v = v0[i], k = k0[key ? i : 0];
    v1[i] = v;
    if (key) k1[i] = k;
  }
  if (c.weight && (int)threadIdx.x < x.tokens) c.weight[to * c.page + threadIdx.x] = c.weight[from * c.page + threadIdx.x];
  if (threadIdx.x == 128) c.k_scale[to] = c.k_scale[from];
  if (threadIdx.x == 129) c.v_scale[to] = c.v_scale[from];
}
// Copies, and the entries that are not fresh pages: those of the parent, and none behind the last one.
__global__ __launch_bounds__(256) void fork_copy_kernel(PageArgs a, int head_dim, int table_blocks) {
  if ((int)blockIdx.x >= table_blocks) {
    const int u = blockIdx.x - table_blocks;
    const Copy x = a.copies[u / a.c.hkv];
    if (x.tokens > 0) copy_page(a.c, head_dim, x, u % a.c.hkv);
    return;
  }
  const int per_seq = (a.s.max_pages + 255) / 256, i = blockIdx.x / per_seq, place = blockIdx.x % per_seq * 256 + threadIdx.x;
  if (place >= a.s.max_pages) return;
  const Next x = next_of(a, i);
  int32_t* const to = a.new_pages + (int64_t)i * a.s.max_pages + place;
  if (place < pages_for(a, x.before)) {
    const int32_t page = entry(a, x.parent, place);
    if (place != x.writes || !a.copies[i].copied) *to = page;
  } else if (place >= pages_for(a, x.after)) {
    *to = -1;
  }
}
__global__ __launch_bounds__(256) void compact_copy_kernel(PageArgs a, int head_dim, int table_blocks) {
  const int32_t end = a.n_copies[1];
  if ((int)blockIdx.x < table_blocks) {
    const int64_t all = (int64_t)a.s.n_seqs * a.s.max_pages;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)table_blocks * 256) {
      const int seq = (int)(i / a.s.max_pages), place = (int)(i % a.s.max_pages);
      int32_t page = place < pages_for(a, cached(a, seq)) ? entry(a, seq, place) : -1;
      if (page >= end && !(a.busy && a.busy[page])) page = a.lowest[page];
      a.new_pages[i] = page;
    }
    return;
  }
  const int64_t all = (int64_t)a.n_copies[0] * a.c.hkv;
  for (int64_t u = blockIdx.x - table_blocks; u < all; u += gridDim.x - table_blocks) copy_page(a.c, head_dim, a.copies[u / a.c.hkv], (int)(u % a.c.hkv));
}

// ---- host ---------------------------------------------------------------------------------------------------------
struct PageSpace { size_t held, read, lowest, list, copies, n_copies, bytes; int32_t words; };
PageSpace page_space(const CacheView& c, int64_t n_copies) {
  PageSpace s = {};
  s.words = (int32_t)(((int64_t)c.n_pages + 31) / 32);
  const size_t bytes = pad_to((size_t)c.n_pages, 256), entries = pad_to((size_t)c.n_pages * 4, 256);
  s.read = bytes;
  s.lowest = 2 * bytes;
  s.list = s.lowest + entries;
  s.copies = s.list + entries;
  s.n_copies = s.copies + pad_to((size_t)n_copies * sizeof(Copy), 256);
  s.bytes = s.n_copies + 256;
  return s;
}
// Whether one block marks and plans.
bool small_call(const CacheView& c, int32_t n_seqs, int32_t max_pages, int32_t n_new) {
  return c.n_pages <= kLdsPages && n_seqs <= kLdsSeqs && (int64_t)n_seqs * max_pages <= kLdsEntries && n_new <= kLdsNew;
}
template <class Kernel>
int launch_small(Kernel kernel, const PageArgs& a, std::atomic<uint64_t>& raised, hipStream_t st) {
  const size_t bytes = lds_bytes(a.words, a.s.n_seqs);
  if (int rc = raise_lds_limit(reinterpret_cast<const void*>(kernel), (int)lds_bytes(kLdsPages / 32, kLdsSeqs), raised)) return rc;
  kernel<<<dim3(1), dim3(kPlanThreads), bytes, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}
void place_scratch(PageArgs& a, const PageSpace& s, void* scratch) {
  char* const at = static_cast<char*>(scratch);
  a.held = reinterpret_cast<uint8_t*>(at);
  a.read = reinterpret_cast<uint8_t*>(at + s.read);
  a.lowest = reinterpret_cast<int32_t*>(at + s.lowest);
  a.list = reinterpret_cast<int32_t*>(at + s.list);
  a.copies = reinterpret_cast<Copy*>(at + s.copies);
  a.n_copies = reinterpret_cast<int32_t*>(at + s.n_copies);
  a.words = s.words;
}
int check_page_sizes(const char* who, const CacheView& c, int32_t n_seqs, int32_t n_new, int32_t max_pages) {
  if (int rc = check_sizes(who, c, n_seqs, max_pages, 0)) return rc;
  if (int rc = check_sizes(who, c, n_new, max_pages, 0)) return rc;
  if (!fits_axis((((int64_t)n_seqs + n_new) * ((max_pages + 63) / 64) + 3) / 4, 256) || !fits_axis((int64_t)n_new * (c.hkv + (max_pages + 255) / 256), 256))
    return fail(FCP_ERR_UNSUPPORTED, "%s: 2^24 blocks of work or more", who);
  // (the pages that new sequences need are added up in 32 bits: at most one for each entry)
  if ((int64_t)n_new * max_pages > INT32_MAX) return fail(FCP_ERR_UNSUPPORTED, "%s: new tables of 2^31 entries or more", who);
  return FCP_OK;
}
int check_scratch(const char* who, const void* scratch, size_t have, size_t need) {
  if (!scratch || (uintptr_t)scratch % 256) return fail(FCP_ERR_INVALID_ARG, "%s: scratch must be 256-byte aligned", who);
  if (have < need) return fail(FCP_ERR_CAPACITY, "%s: scratch has %zu bytes, %zu are needed", who, have, need);
  return FCP_OK;
}

}  // namespace

// 0: refused
size_t page_scratch_bytes(const char* who, const CacheView& c, bool fork, int32_t n_seqs, int32_t max_pages) {
  if (check_page_sizes(who, c, fork ? 0 : n_seqs, fork ? n_seqs : 0, max_pages)) return 0;
  return page_space(c, fork ? n_seqs : c.n_pages).bytes;
}

}  // namespace fcp

extern "C" int fcp_cache_fork(const fcp_cache* cache, const int32_t* pages, const int32_t* kv_len, int32_t n_seqs, int32_t max_pages, const int32_t* parent,
                              const int32_t* news, int32_t n_new, const uint8_t* busy, int32_t* new_pages, int32_t* new_len, int32_t* counts,
                              void* scratch, size_t scratch_bytes, void* stream) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_cache_fork";
  PageArgs a = {};
  if (int rc = check_cache(who, cache, false, &a.c)) return rc;
  if (int rc = check_page_sizes(who, a.c, n_seqs, n_new, max_pages)) return rc;
  if (int rc = check_seqs(who, a.c, nullptr, false, kv_len, pages, n_seqs, max_pages, 0)) return rc;
  if (!counts || (n_new > 0 && (!parent || !news || !new_len || (max_pages > 0 && !new_pages)))) return fail(FCP_ERR_INVALID_ARG, "%s: null argument", who);
  if (int rc = check_int_pointers(who, {pages, kv_len, parent, news, new_pages, new_len, counts})) return rc;
  const PageSpace space = page_space(a.c, n_new);
  if (int rc = check_scratch(who, scratch, scratch_bytes, space.bytes)) return rc;
  const int64_t row = (int64_t)4 * max_pages;
  if (int rc = check_apart(who, {{new_pages, n_new * row}, {new_len, (int64_t)4 * n_new}, {counts, 12}, {scratch, (int64_t)space.bytes}},
                           {{pages, n_seqs * row}, {kv_len, (int64_t)4 * n_seqs}, {parent, (int64_t)4 * n_new}, {news, (int64_t)4 * n_new}, {busy, a.c.n_pages}}))
    return rc;
  a.s = {nullptr, kv_len, pages, n_seqs, max_pages, 0};
  a.parent = parent;
  a.news = news;
  a.n_new = n_new;
  a.busy = busy;
  a.new_pages = new_pages;
  a.new_len = new_len;
  a.counts = counts;
  place_scratch(a, space, scratch);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (small_call(a.c, n_seqs, max_pages, n_new)) {
    static std::atomic<uint64_t> raised;
    if (int rc = launch_small(fork_small_kernel, a, raised, st)) return rc;
  } else {
    clear_kernel<true><<<dim3((unsigned)((max((a.c.n_pages + 3) / 4, n_new) + 255) / 256)), dim3(256), 0, st>>>(a);
    FCP_HIP_CHECK(hipGetLastError());
    const int64_t units = ((int64_t)n_seqs + n_new) * ((max_pages + 63) / 64);
    if (units > 0) {
      mark_kernel<true><<<dim3((unsigned)((units + 3) / 4)), dim3(256), 0, st>>>(a);
      FCP_HIP_CHECK(hipGetLastError());
    }
    fork_plan_kernel<<<dim3(1), dim3(kPlanThreads), 0, st>>>(a);
    FCP_HIP_CHECK(hipGetLastError());
  }
  if (n_new > 0) {
    const int64_t tables = (int64_t)n_new * ((max_pages + 255) / 256);
    fork_copy_kernel<<<dim3((unsigned)(tables + (int64_t)n_new * a.c.hkv)), dim3(256), 0, st>>>(a, cache->head_dim, (int)tables);
    FCP_HIP_CHECK(hipGetLastError());
  }
  return FCP_OK;
}

extern "C" int fcp_cache_compact(const fcp_cache* cache, const int32_t* pages, const int32_t* kv_len, int32_t n_seqs, int32_t max_pages, const uint8_t* busy,
                                 int32_t* new_pages, int32_t* counts, void* scratch, size_t scratch_bytes, void* stream) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_cache_compact";
  PageArgs a = {};
  if (int rc = check_cache(who, cache, false, &a.c)) return rc;
  if (int rc = check_page_sizes(who, a.c, n_seqs, 0, max_pages)) return rc;
  if (int rc = check_seqs(who, a.c, nullptr, false, kv_len, pages, n_seqs, max_pages, 0)) return rc;
  if (!counts || (n_seqs > 0 && max_pages > 0 && !new_pages)) return fail(FCP_ERR_INVALID_ARG, "%s: null argument", who);
  if (int rc = check_int_pointers(who, {pages, kv_len, new_pages, counts})) return rc;
  const PageSpace space = page_space(a.c, a.c.n_pages);
  if (int rc = check_scratch(who, scratch, scratch_bytes, space.bytes)) return rc;
  const int64_t tables = (int64_t)4 * n_seqs * max_pages;
  const Span old = {new_pages == pages ? nullptr : pages, tables};       // (the new tables may be the old ones)
  if (int rc = check_apart(who, {{new_pages, tables}, {counts, 12}, {scratch, (int64_t)space.bytes}}, {old, {kv_len, (int64_t)4 * n_seqs}, {busy, a.c.n_pages}})) return rc;
  a.s = {nullptr, kv_len, pages, n_seqs, max_pages, 0};
  a.busy = busy;
  a.new_pages = new_pages;
  a.counts = counts;
  place_scratch(a, space, scratch);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t entries = (int64_t)n_seqs * max_pages;
  if (small_call(a.c, n_seqs, max_pages, 0)) {
    static std::atomic<uint64_t> raised;
    if (int rc = launch_small(compact_small_kernel, a, raised, st)) return rc;
  } else {
    clear_kernel<false><<<dim3((unsigned)(((a.c.n_pages + 3) / 4 + 255) / 256)), dim3(256), 0, st>>>(a);
    FCP_HIP_CHECK(hipGetLastError());
    const int64_t units = (int64_t)n_seqs * ((max_pages + 63) / 64);
    if (units > 0) {
      mark_kernel<false><<<dim3((unsigned)((units + 3) / 4)), dim3(256), 0, st>>>(a);
      FCP_HIP_CHECK(hipGetLastError());
    }
    compact_plan_kernel<<<dim3(1), dim3(kPlanThreads), 0, st>>>(a);
    FCP_HIP_CHECK(hipGetLastError());
  }
  const int table_blocks = (int)min((entries + 1023) / 1024, (int64_t)256), copy_blocks = (int)min(min((int64_t)a.c.n_pages, entries) * a.c.hkv, (int64_t)2048);
  if (entries > 0) {
    compact_copy_kernel<<<dim3((unsigned)(table_blocks + copy_blocks)), dim3(256), 0, st>>>(a, cache->head_dim, table_blocks);
    FCP_HIP_CHECK(hipGetLastError());
  }
  return FCP_OK;
}
