// Paged key-value caches: what lsa_kv_append and lsa_paged_attn share.
//
// lsa_paged_attn deals the key tiles of all sequences out evenly: they form one list, ordered by (sequence, block of KV heads,
// position), and unit u of the grid takes entries [u * per, (u + 1) * per).  Lengths differ by orders of magnitude between sequences,
// and a grid by sequence would wait for the longest.  Every unit, and the kernel that joins the parts, derives the same list from ctx_len.
#pragma once

#include "lsa_common.cuh"
#include "lsa_internal.h"

namespace lsa {
namespace paged {

constexpr float kLog2e = 1.4426950408889634f;

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

__device__ __forceinline__ SeqTiles seq_tiles(const PagedAttnArgs& a, int b, int shift) {
  SeqTiles t;
  t.n = seq_length(a, b);
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

// The list: its length, the entries of a unit, and how many entries lie before sequence b.
struct List {
  int64_t total, per;
};
// By a whole warp.  `before` (optional): entries of the sequences below b_before.
__device__ __forceinline__ int64_t warp_sum(int64_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ List list_of(int64_t total, const PagedAttnArgs& a) {
  const int64_t even = (total + a.units - 1) / a.units;
  return {total, even > a.min_tiles ? even : a.min_tiles};
}

// Where a unit's entries begin.
struct Cursor {
  int b, block, tile;   // sequence, block of KV heads, tile
  int64_t left;         // entries of the unit from here on
  SeqTiles st;
};
// By a whole warp: unit u's first entry.  Each lane counts a run of consecutive sequences.
__device__ __forceinline__ Cursor first_entry(const PagedAttnArgs& a, int unit, int shift, int blocks, int lane) {
  const int run = (a.batch + 31) / 32;
  int64_t mine = 0;
  for (int i = 0; i < run; ++i) {
    const int b = lane * run + i;
    if (b < a.batch) mine += seq_tiles(a, b, shift).count;
  }
  int64_t upto = mine;   // inclusive scan
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  const List l = list_of(__shfl_sync(0xffffffffu, upto, 31) * blocks, a);
  Cursor c{};
  const int64_t t0 = unit * l.per;
  if (t0 >= l.total) return c;
  c.left = min64(l.per, l.total - t0);
  const unsigned past = __ballot_sync(0xffffffffu, upto * blocks > t0);
  const int owner = __ffs(past) - 1;
  int64_t base = __shfl_sync(0xffffffffu, upto - mine, owner) * blocks;
  c.b = owner * run;
  c.st = seq_tiles(a, c.b, shift);
  while (base + static_cast<int64_t>(c.st.count) * blocks <= t0) {
    base += static_cast<int64_t>(c.st.count) * blocks;
    c.st = seq_tiles(a, ++c.b, shift);
  }
  const int64_t off = t0 - base;
  c.block = static_cast<int>(off / c.st.count);
  c.tile = static_cast<int>(off % c.st.count);
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

}  // namespace paged
}  // namespace lsa
