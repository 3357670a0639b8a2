// Paged key-value caches: what lsa_kv_append and lsa_paged_attn share.
//
// lsa_paged_attn deals the key tiles of all sequences out evenly: they form one list, ordered by (sequence, block of KV heads,
// position), and unit u of the grid (a block per SM) takes entries [u * per, (u + 1) * per).  Lengths differ by orders of magnitude
// between sequences, and a grid by sequence would wait for the longest.  Every unit derives the same list from ctx_len and leaves word of
// what there is to join, so the host needs no lengths and a captured call stays right as they grow.
#pragma once

#include "lsa_common.cuh"
#include "lsa_internal.h"

namespace lsa {
namespace paged {

constexpr float kLog2e = 1.4426950408889634f;

// Weights are 2^(score - reference), and a head's reference is moved only when its maximum has grown by more than 2^8, so that the
// output is rarely rescaled: a weight is at most 2^8 where the reference was the maximum.  fp16 weights end at 2^-24, and a long
// sequence may have its mass in hundreds of thousands of weights smaller than that beside one of 1, so their reference lies 2^7 below
// the maximum: weights of at most 2^15, and down to 2^-32 of the largest.  (bf16 has the range of fp32.)
constexpr float kRescaleGap = 8.f;
template <bool kF16Weights>
constexpr float kLift = kF16Weights ? 7.f : 0.f;

// A number of the caller's that points outside its array: recorded in the notice word (see lsa_status), never followed.
__device__ __forceinline__ void report_index(int* notice) { report_status(notice, kDevBadIndex); }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The tiles of one sequence: those of the sink, then those of the window (all of them where nothing is hidden).
struct SeqTiles {
  int n, lo, sink;        // key s is seen iff s < n and (s >= lo or s < sink)
  int head, skip, count;  // tile i starts at key (i < head ? i : i + skip) << shift
  __device__ __forceinline__ int first_key(int i, int shift) const { return (i < head ? i : i + skip) << shift; }
  __device__ __forceinline__ bool seen(int s) const { return s < n && (s >= lo || s < sink); }
  // keys s .. s + len - 1: whether any, and whether all of them are seen
  __device__ __forceinline__ bool any_seen(int s, int len) const { return s < n && (s + len > lo || s < sink); }
  __device__ __forceinline__ bool all_seen(int s, int len) const { return s + len <= n && (s >= lo || s + len <= sink); }
};

__device__ __forceinline__ int seq_length(const PagedAttnArgs& a, int b, bool report = false) {
  const int n = a.ctx_len[b];
  if (n < 0 || n > a.max_len) {
    if (report) report_index(a.notice);
    return n < 0 ? 0 : a.max_len;
  }
  return n;
}

__device__ __forceinline__ SeqTiles tiles_of(const PagedAttnArgs& a, int n, int shift) {
  SeqTiles t;
  t.n = n;
  const int all = (t.n + (1 << shift) - 1) >> shift;
  if (a.window <= 0 || t.n <= static_cast<int64_t>(a.sink) + a.window) {
    t.lo = t.sink = t.head = t.skip = 0;
    t.count = all;
  } else {
    t.lo = t.n - a.window;
    t.sink = a.sink;
    t.head = (a.sink + (1 << shift) - 1) >> shift;
    const int w0 = max(t.head, t.lo >> shift);
    t.skip = w0 - t.head;
    t.count = all - t.skip;
  }
  return t;
}

__device__ __forceinline__ SeqTiles seq_tiles(const PagedAttnArgs& a, int b, int shift) { return tiles_of(a, seq_length(a, b), shift); }

// Where a unit is in the list.
struct Cursor {
  int b, block, tile;   // sequence, block of KV heads, tile
  int left;             // entries of the unit from here on
  int per, near;        // see first_entry
  SeqTiles st;
};
// By a whole warp: unit u's first entry.  The list is cut every `per` entries, and a cut no more than `near` from an end of its (sequence,
// block) is moved there: a tile more costs a unit less than a part that has to be written and joined.
// (The list has fewer than 2^31 entries: the host sees to that.)
__device__ __forceinline__ Cursor first_entry(const PagedAttnArgs& a, int unit, int shift, int blocks, int lane) {
  const int run = (a.batch + 31) / 32;   // each lane counts a run of consecutive sequences
  int mine = 0, n = 0;
  for (int i = 0; i < run; ++i) {
    const int b = lane * run + i;
    if (b < a.batch) {
      n = seq_length(a, b);
      mine += tiles_of(a, n, shift).count;
    }
  }
  mine *= blocks;
  int upto = mine;   // inclusive scan
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  const int total = __shfl_sync(0xffffffffu, upto, 31);
  Cursor c{};
  // (down to one tile each, though every part has to be joined: at least two took 11.8 us instead of 11.3 for one latent sequence of 300
  // tokens, 17.2 instead of 13.0 for four of 777, and 9.5 instead of 9.3 for one of 2000 with 8 KV heads)
  c.per = (total - 1) / a.units + 1;
  c.near = min(a.near, c.per - 1);
  const int64_t t0 = static_cast<int64_t>(unit) * c.per;
  if (t0 >= total) return c;
  auto locate = [&](int at) {   // entry `at`
    const int owner = __ffs(__ballot_sync(0xffffffffu, upto > at)) - 1;
    int off = at - __shfl_sync(0xffffffffu, upto - mine, owner);
    c.b = owner * run;
    c.block = 0;
    if (run == 1) {   // (the owner has the length: a load less on the way to the first tile)
      c.st = tiles_of(a, __shfl_sync(0xffffffffu, n, owner), shift);
    } else {
      c.st = seq_tiles(a, c.b, shift);
      while (c.st.count * blocks <= off) {
        off -= c.st.count * blocks;
        c.st = seq_tiles(a, ++c.b, shift);
      }
    }
    while (off >= c.st.count) {   // (`blocks` is small)
      off -= c.st.count;
      ++c.block;
    }
    c.tile = off;
  };
  auto cut = [&](int at) -> int {   // where the cut before entry `at` comes to lie
    locate(at);
    const int rest = c.st.count - c.tile;
    return min(c.tile, rest) > c.near ? at : c.tile <= rest ? at - c.tile : at + rest;
  };
  const int first = static_cast<int>(t0), next = first + min(c.per, total - first);
  if (c.near == 0) {
    c.left = next - first;
    locate(first);
    return c;
  }
  const int end = next < total ? cut(next) : total, start = cut(first);
  c.left = end - start;
  if (c.left > 0 && start != first) locate(start);
  return c;
}
// The next entry; true: it belongs to another (sequence, block).
__device__ __forceinline__ bool advance(const PagedAttnArgs& a, Cursor& c, int shift, int blocks) {
  --c.left;
  if (++c.tile < c.st.count) return false;
  c.tile = 0;
  if (++c.block < blocks) return true;
  c.block = 0;
  if (c.left > 0) {
    do c.st = seq_tiles(a, ++c.b, shift);
    while (c.st.count == 0);
  }
  return true;
}

// What a unit leaves behind: its first (sequence, block) in slot 2u of the partial results if that began or goes on in another
// unit, its last in slot 2u + 1 if that is another one and goes on in the next.  Whoever holds the beginning of one that goes on
// says so for the kernel that joins the parts: {parts, sequence, block, slot of the first part}; the others are the slots
// 2 (u + 1), 2 (u + 2), ...
__device__ __forceinline__ void say_parts(const PagedAttnArgs& a, int unit, const Cursor& last, bool begins_here, bool first) {
  const int rest = last.st.count - (last.tile + 1);
  const bool goes_on = begins_here && rest > 0;
  a.parts[unit] = make_int4(goes_on ? 1 + (rest - last.near + last.per - 1) / last.per : 0, last.b, last.block, 2 * unit + (first ? 0 : 1));
}

// ---- the kernels that join parts: what a block has to do.
// The units' words about their parts (148 numbers, whatever the batch) give each owner (a unit that holds a beginning) a number of rounds; round `it` of all of them is
// looked up by the threads together.
constexpr int kJoinThreads = 256;
struct JoinList {
  int warp_sum[kJoinThreads / 32];
  int4 own;        // of the round at hand: {parts, sequence, block, slot of the first part}
  int unit, round;
};
// By all kJoinThreads threads.  rounds_of(parts, owners): rounds of an owner.  begins: rounds before this thread's unit; returns all rounds.
template <class F>
__device__ __forceinline__ int join_list(const PagedAttnArgs& a, JoinList& s, int tid, int4* mine, int* begins, int* owners, F rounds_of) {
  static_assert(kMaxPagedUnits <= kJoinThreads, "a thread per unit");
  const int lane = tid & 31, warp = tid >> 5;
  *mine = tid < a.units ? __ldcg(a.parts + tid) : make_int4(0, 0, 0, 0);
  // (units that gave up on a wait have left nothing, and nothing said about it)
  const bool raised = a.status != nullptr && *reinterpret_cast<const volatile int*>(a.status) != 0;
  *owners = __syncthreads_count(mine->x > 0);
  const int x = rounds_of(mine->x, *owners);
  int upto = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) s.warp_sum[warp] = upto;
  if (__syncthreads_or(raised)) return 0;
  int before = 0, total = 0;
#pragma unroll
  for (int i = 0; i < kJoinThreads / 32; ++i) {
    const int w = s.warp_sum[i];
    if (i < warp) before += w;
    total += w;
  }
  *begins = before + upto - x;
  return total;
}
// The owner of round `it`, for all threads (it < all rounds).
template <class F>
__device__ __forceinline__ void join_find(JoinList& s, int tid, int it, const int4& mine, int begins, int owners, F rounds_of) {
  __syncthreads();   // (the round before has been worked on)
  if (it >= begins && it < begins + rounds_of(mine.x, owners)) {
    s.own = mine;
    s.unit = tid;
    s.round = it - begins;
  }
  __syncthreads();
}

}  // namespace paged
}  // namespace lsa
