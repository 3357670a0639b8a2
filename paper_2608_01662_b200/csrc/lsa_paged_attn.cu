// lsa_paged_attn for caches with separate keys and values: one query per sequence, up to 16 query heads per KV head.
//
// A query head's 64 or 128 dims meet each cached key and value once: at most 16 flop per byte read (32 where it is a code), so the
// kernel has to keep HBM busy and everything else has to stay out of its way.  Both products are m16n8k16 MMAs with the cache as the A operand and the
// heads as the eight columns: S^T = K Q^T (16 tokens x 8 heads) and O^T = V^T P^T (16 dims x 8 heads).  The other way round the
// heads are 16 rows, of which groups of 4 or 8 heads leave most empty: twice the MMAs and twice the registers of O.
//
// A tile is eight strips of 16 or 32 tokens of one KV head each: all KV heads of a block (up to eight; a row of the cache is then read
// whole) times as many strips as make up eight.  One warp copies tiles by TMA, a box per cache page, keys and values (32 KB
// each) in turn, into a ring of six slots; eight warps take a strip of every tile each and keep reference, sum and output of
// their strips in registers, so that they meet only at the end of a sequence.  (With the copies issued by the warps that use
// them, half of the instructions were the bookkeeping of rings and pages: 400 per strip of 16 tokens where the products take 50;
// 16 heads over one KV head, 783 thousand tokens: 82 us, so 74.)
//
// Measured: 128 sequences of up to 7000 tokens, 8 KV heads of 128, 196 us (6.3 TB/s, 0.96 of a copy's rate); the one KV head above
// 74 us (0.83: the SMs end up to 15 % apart, whole GPCs get less of HBM's rate, and handing out the end of the list by a ticket cost more than
// that: 91 us).  Short sequences take 8 to 10 us: 4 until the first tile is there, the rest its work and the kernel that joins.
//
// e4m3 caches: a code is exact in fp16, and so is a query scaled by a power of two of its own head, so the scores' products
// are fp16 MMAs of codes and the scale of a key is applied to the score.  A value's scale is applied to its weight; the product, times a
// power of two of its head's own that follows the largest of them, is rounded to fp16: scales of any size, and what lies 2^-21 below
// the largest product still has all its bits.  (With weights times scales in bf16 and codes turned into bf16 139 to 146 us instead
// of 137, and a third more error.)  The conversions of codes keep these caches at 0.86 of a copy's rate (32 sequences of up to 32
// thousand tokens, 64 query and 8 KV heads, 774 MB in 137 us).
//
// 9 to 16 query heads per KV head are two groups of columns, the products and the softmax of each strip twice; that shows most where a
// strip is few bytes: 99 thousand tokens of 128 over 8 heads 83 us in bf16 (0.75 of a copy's rate), 70 as codes (0.45); 688 thousand of
// 16 over 1 head 42 us with 64 dims in bf16 (0.64), 68 with 128 dims as codes (0.41; there 60 to 92 bytes a thread do not fit the 168
// registers).
#include "lsa_paged.cuh"
#include "lsa_tc.cuh"

namespace lsa {

namespace {

using paged::Cursor;
using paged::exp2_fast;

constexpr int kWarps = 8, kThreads = 32 * (kWarps + 1);   // and the one that copies
constexpr int kRing = 6;

template <int V>
struct IntC { static constexpr int value = V; };

// kTiles: groups of eight query heads per KV head (1 or 2).
template <int D, bool kE4M3, int kTiles>
struct Shape {
  static constexpr int kRowBytes = D * (kE4M3 ? 1 : 2);            // of a head
  static constexpr int kBlockBytes = kRowBytes < 128 ? 64 : 128;   // columns of a TMA box lie in blocks of this many bytes
  static constexpr int kBlocks = kRowBytes / kBlockBytes;          // of a head
  static constexpr int kRows = kRowBytes == 256 ? 16 : 32, kRowShift = kRows == 32 ? 5 : 4;   // of a strip
  static constexpr int kBytes = kWarps * kRows * kRowBytes;        // of a tile's keys, and of its values: one slot each
  static constexpr int kScales = kE4M3 ? kWarps * kRows * 4 : 0;
  static constexpr int kMergeDims = kTiles == 2 ? 32 : 64;   // dims that are put together at a time: what there is room for
  static constexpr int kMergePitch = kMergeDims + 2;               // floats
  static constexpr int kMerge = kWarps * 8 * kTiles * kMergePitch * 4;
  static constexpr int kSmem = 1024 + kRing * (kBytes + kScales) + kMerge + kWarps * 8 * kTiles * 8 + 2 * kRing * 8;
};

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool kF16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (kF16) mma_f16(d, a, b0, b1);
  else mma_bf16(d, a, b0, b1);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
// Transposes an 8x8 matrix of 16-bit elements held as an MMA fragment.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint16_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(two));
  return r;
}
template <int kBytes>
__device__ __forceinline__ void cp_async_ca(uint32_t dst, const void* src, int src_bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;\n" ::"r"(dst), "l"(src), "n"(kBytes), "r"(src_bytes));
}
// The barrier counts this thread once its earlier cp.async have landed (its count includes the arrival).
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) { asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void workers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory"); }

// heads_shift: log2 of the KV heads that a block works on at the same time (8, 4, 2 or 1, a divisor of G).
template <typename T, int D, bool kE4M3, int kTiles>
__global__ void __launch_bounds__(kThreads, 1)
paged_attn_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, PagedAttnArgs p, int heads_shift) {
  using S = Shape<D, kE4M3, kTiles>;
  constexpr bool kF16 = !__is_same(T, __nv_bfloat16);
  constexpr bool k16 = kF16 || kE4M3;   // both products of fp16 numbers
  constexpr float kLift = paged::kLift<kF16 && !kE4M3>, kGap = paged::kRescaleGap + kLift;
  constexpr int R = S::kRows, kSub = R / 16, kHeadsOf = 8 * kTiles;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  float* const scales = reinterpret_cast<float*>(ring + kRing * S::kBytes);     // [slot][row of the tile][head]
  float* const merge = scales + kRing * S::kScales / 4;
  float2* const ml = reinterpret_cast<float2*>(merge + S::kMerge / 4);          // {reference, sum} per warp and head
  const uint32_t full = smem_u32(ml + kWarps * kHeadsOf), empty = full + 8 * kRing;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int strip_shift = 3 - heads_shift, n_strips = 1 << strip_shift;
  const int shift = S::kRowShift + strip_shift;     // keys of a tile
  const int blocks = p.G >> heads_shift;
  const int box_shift = min(shift, p.page_shift);   // keys of a box

  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    for (int i = 0; i < kRing; ++i) {
      tc::mbar_init(full + 8 * i, kE4M3 ? 33 : 1);
      tc::mbar_init(empty + 8 * i, kWarps);
    }
    tc::fence_mbar_init();
  }
  pdl_wait();
  pdl_launch_dependents();
  const bool raised = tc::status_raised(p.status);
  Cursor cur = paged::first_entry(p, blockIdx.x, shift, blocks, lane);
  const bool dead = __syncthreads_or(raised) != 0;   // the same in all threads
  if (dead) return;

  if (warp == kWarps) {
    // ================= copies =================
    const int page_mask = (1 << p.page_shift) - 1;
    const int beyond = static_cast<int>(static_cast<int64_t>(max(p.n_pages, 1)) << p.page_shift);   // the first row past the pool: rows of zeros
    const int box_bytes = (S::kBytes >> shift) << box_shift;   // (a tile's bytes over its keys, times a box's)
    const int n_boxes = 1 << (shift - box_shift);
    // scales of consecutive rows follow one another where a block has all heads: 16 bytes a copy; else 2^copy_shift heads of a row
    // (155 sequences of 1640 tokens, one KV head, pages of 16, by rows and boxes: 41.4 us; so: 22.3)
    const int copy_shift = blocks == 1 ? 2 : min(heads_shift, 2);
    // a lane's box of the tile at the cursor: its cache row; past the pool if its page is not one, -1 if nobody sees its keys
    auto row_of = [&]() -> int {
      if (cur.left <= 0 || lane >= n_boxes) return -1;
      const int s0 = cur.st.first_key(cur.tile, shift) + (lane << box_shift);
      if (!cur.st.any_seen(s0, 1 << box_shift)) return -1;
      const int page = p.page_table[cur.b * p.pt_stride + (s0 >> p.page_shift)];
      if (page < 0 || page >= p.n_pages) {
        paged::report_index(p.notice);
        return beyond;
      }
      return (page << p.page_shift) + (s0 & page_mask);
    };
    int row = row_of(), slot = 0;
    uint32_t use = 0;
    const int entries = cur.left;
    int issued = 0;
    bool alive = true;
    for (int g = 0; g < entries && alive; ++g) {
      const int this_row = row, head0 = cur.block << heads_shift;
      paged::advance(p, cur, shift, blocks);
      row = row_of();   // (its page number is on its way while this tile waits for its slots)
      const int n_here = __popc(__ballot_sync(0xffffffffu, this_row >= 0));
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        alive = alive && __all_sync(0xffffffffu, tc::mbar_wait(empty + 8 * slot, use ^ 1u, p.status));
        if (!alive) break;
        const uint32_t bar = full + 8 * slot;
        if (lane == 0) tc::mbar_expect_tx(bar, static_cast<uint32_t>(n_here * box_bytes));
        __syncwarp();
        if (this_row >= 0)
          tc::tma_load_3d(smem_u32(ring) + slot * S::kBytes + lane * box_bytes, kv == 0 ? &k_map : &v_map, 0, this_row, head0 * S::kBlocks, bar);
        if constexpr (kE4M3) {
          const float* src = kv == 0 ? p.k_scale : p.v_scale;
          const uint32_t dst = smem_u32(scales) + slot * S::kScales;
          auto fetch = [&](auto floats_c) {   // so many floats a copy
            constexpr int kFloats = decltype(floats_c)::value;
#pragma unroll
            for (int i = 0; i < kWarps * R / kFloats / 32; ++i) {
              const int f = (32 * i + lane) * kFloats, r = f >> heads_shift;   // the copy's first float in the slot, its row
              const int r0 = __shfl_sync(0xffffffffu, this_row, r >> box_shift);
              const bool there = r0 < beyond;
              const float* s = src + (there ? static_cast<int64_t>(r0 + (r & ((1 << box_shift) - 1))) * p.G + head0 + (f & ((1 << heads_shift) - 1)) : 0);
              if (r0 >= 0) cp_async_ca<4 * kFloats>(dst + 4 * f, s, there ? 4 * kFloats : 0);
            }
          };
          if (copy_shift == 2) fetch(IntC<4>{});
          else if (copy_shift == 1) fetch(IntC<2>{});
          else fetch(IntC<1>{});
          cp_async_arrive(bar);
        }
        __syncwarp();
        ++issued;
        if (++slot == kRing) {
          slot = 0;
          use ^= 1u;
        }
      }
    }
    // every copy has landed before the block ends, also if somebody gave up on a wait
    for (int i = max(issued - kRing, 0); i < issued; ++i) (void)tc::mbar_wait(full + 8 * (i % kRing), static_cast<uint32_t>(i / kRing) & 1u, nullptr);
    return;
  }

  // ================= strips =================
  const int g4 = lane >> 2, t4 = lane & 3;
  const int head_l = warp >> strip_shift, strip = warp & (n_strips - 1);
  const int group = p.H / p.G;
  if (cur.left == 0 && tid == 0) p.parts[blockIdx.x] = make_int4(0, 0, 0, 0);

  // Where the strip lies in a slot: boxes of [block of columns][key][block bytes], 16-byte units XORed as TMA does it, which also keeps the
  // eight rows that an ldmatrix phase reads in different banks.  A strip of 32 tokens in pages of 16 lies in two boxes.
  const int block_stride = S::kBlockBytes << box_shift;
  auto strip_at = [&](int key) -> uint32_t {   // offset of a key of the strip, first block of the head
    const int k = strip * R + key, j = k >> box_shift, in = k & ((1 << box_shift) - 1);
    return j * (block_stride * S::kBlocks << heads_shift) + head_l * S::kBlocks * block_stride + in * S::kBlockBytes;
  };
  // XOR of the unit index of row r; (rows of a strip are aligned to 16)
  auto twist = [](int r) -> uint32_t { return S::kBlockBytes == 64 ? ((r >> 1) & 3) << 4 : (r & 7) << 4; };
  // Addresses of a lane in a slot (without the slot's base), unit 0 or 1: units 2 i and 2 i + 1 further on are an XOR of 32 i.
  uint32_t k_off[kSub], v_off[kSub];
  if constexpr (!kE4M3) {
#pragma unroll
    for (int j = 0; j < kSub; ++j) {
      const int rk = 16 * j + (lane & 15), rv = 16 * j + (lane & 7) + ((lane >> 4) << 3);
      k_off[j] = strip_at(rk) + (static_cast<uint32_t>(lane >> 4) << 4 ^ twist(rk));
      v_off[j] = strip_at(rv) + (static_cast<uint32_t>((lane >> 3) & 1) << 4 ^ twist(rv));
    }
  } else {   // one row of codes per lane, keys and values alike
    k_off[0] = v_off[0] = strip_at(lane) + twist(lane);
  }

  // ---- the state of a (sequence, block): query fragments, output, references and sums of the heads 8 n + 2 t4, + 1
  uint32_t qf[kTiles][D / 16][2];
  float o[kTiles][D / 16][4];
  float zs[kTiles][2], m_used[kTiles][2], l_run[kTiles][2];
  // e4m3: the output is of weights times value scales, times 2^k of their own per head: w_up = 2^k, set so that w_max, the largest of
  // them so far when it was set, came to 2^7
  float w_max[kTiles][2], w_up[kTiles][2];
  auto up_of = [](float w) { return __uint_as_float(static_cast<uint32_t>(min(261 - static_cast<int>(__float_as_uint(w) >> 23), 253)) << 23); };
  auto begin = [&]() {
    const int head0 = ((cur.block << heads_shift) + head_l) * group;
    const T* q = static_cast<const T*>(p.q) + cur.b * p.ld_q + static_cast<int64_t>(head0) * D;
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      const bool on = 8 * n + g4 < group;
      const uint32_t* row = reinterpret_cast<const uint32_t*>(q + (on ? 8 * n + g4 : 0) * D);   // pairs of dims
      zs[n][0] = zs[n][1] = p.scale2;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        if constexpr (!kE4M3) {
          qf[n][k][0] = on ? row[8 * k + t4] : 0u;
          qf[n][k][1] = on ? row[8 * k + 4 + t4] : 0u;
        } else {   // dims 16 k + 4 t .. + 3 take the places of the rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9 of step k
          const uint2 w = on ? *reinterpret_cast<const uint2*>(row + 8 * k + 2 * t4) : make_uint2(0u, 0u);
          qf[n][k][0] = w.x;
          qf[n][k][1] = w.y;
        }
      }
      if constexpr (kE4M3 && !kF16) {
        float top = 0.f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&qf[n][k][h]));
            top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
          }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // largest element in [2^14, 2^15): what lies 2^-29 below it still has all its bits
        const int sh = e5m2_head_shift(top);
        const float up = __uint_as_float(static_cast<uint32_t>(127 + sh) << 23), down = __uint_as_float(static_cast<uint32_t>(127 - sh) << 23);
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&qf[n][k][h]));
            qf[n][k][h] = pack_f16(f.x * up, f.y * up);
          }
        // (not 0, however small: a hidden key's -inf times that is not -inf)
        zs[n][0] = fmaxf(zs[n][0] * __shfl_sync(0xffffffffu, down, 8 * t4), 0x1p-149f);
        zs[n][1] = fmaxf(zs[n][1] * __shfl_sync(0xffffffffu, down, 8 * t4 + 4), 0x1p-149f);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        m_used[n][c] = -INFINITY;
        l_run[n][c] = 0.f;
        w_max[n][c] = 0.f;
        w_up[n][c] = up_of(0.f);
      }
#pragma unroll
      for (int i = 0; i < D / 16; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
    }
  };

  int slot = 0;
  uint32_t use = 0;
  bool ok = true;
  auto arrived = [&]() {   // the next slot's bytes are there
    if (ok) ok = __all_sync(0xffffffffu, tc::mbar_wait(full + 8 * slot, use, p.status));
  };
  auto release = [&]() {
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(empty + 8 * slot);
    if (++slot == kRing) {
      slot = 0;
      use ^= 1u;
    }
  };

  // ---- one strip
  auto work = [&]() {
    const int s0 = cur.st.first_key(cur.tile, shift) + strip * R;
    const bool any = cur.st.any_seen(s0, R), partial = !cur.st.all_seen(s0, R);
    arrived();
    if (!any) {   // (the slots are waited for and given free all the same: a warp ahead of the others would be counted twice)
      release();
      arrived();
      release();
      return;
    }
    float s[kSub][kTiles][4];
#pragma unroll
    for (int j = 0; j < kSub; ++j)
#pragma unroll
      for (int n = 0; n < kTiles; ++n) s[j][n][0] = s[j][n][1] = s[j][n][2] = s[j][n][3] = 0.f;
    {
      const uint32_t kb = smem_u32(ring) + slot * S::kBytes;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        if constexpr (!kE4M3) {
#pragma unroll
          for (int j = 0; j < kSub; ++j) {
            uint32_t w[4];
            ldmatrix_x4(w, (kb + k_off[j] + (k >> 2) * block_stride) ^ ((k & 3) * 32));
#pragma unroll
            for (int n = 0; n < kTiles; ++n) mma<k16>(s[j][n], w, qf[n][k][0], qf[n][k][1]);
          }
        } else {
          uint32_t c[4];   // four codes of a key: dims 16 k + 4 t .. + 3 of keys 8 i + lane / 4
          ldmatrix_x4(c, (kb + k_off[0]) ^ (k * 16));
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t w[4] = {e4m3x2_to_f16x2(static_cast<uint16_t>(c[2 * j])), e4m3x2_to_f16x2(static_cast<uint16_t>(c[2 * j + 1])),
                                   e4m3x2_to_f16x2(static_cast<uint16_t>(c[2 * j] >> 16)), e4m3x2_to_f16x2(static_cast<uint16_t>(c[2 * j + 1] >> 16))};
#pragma unroll
            for (int n = 0; n < kTiles; ++n) mma<k16>(s[j][n], w, qf[n][k][0], qf[n][k][1]);
          }
        }
      }
    }
    if constexpr (kE4M3) {
      const float* sc = scales + slot * (S::kScales / 4) + ((strip * R + g4) << heads_shift) + head_l;
#pragma unroll
      for (int j = 0; j < kSub; ++j)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float x = sc[(16 * j + 8 * r) << heads_shift];
#pragma unroll
          for (int n = 0; n < kTiles; ++n) {
            s[j][n][2 * r] *= x;
            s[j][n][2 * r + 1] *= x;
          }
        }
    }
    release();
    // the thread's keys are 16 j + g4 and 8 more, its heads 8 n + 2 t4 and the next
    if (partial) {
#pragma unroll
      for (int j = 0; j < kSub; ++j)
#pragma unroll
        for (int r = 0; r < 2; ++r)
          if (!cur.st.seen(s0 + 16 * j + 8 * r + g4)) {
#pragma unroll
            for (int n = 0; n < kTiles; ++n) s[j][n][2 * r] = s[j][n][2 * r + 1] = -INFINITY;
          }
    }
    // P with the references as they are; only where a head has grown too far is its reference moved before
    float mx[kTiles][2];
    bool need = false;
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x = fmaxf(s[0][n][c], s[0][n][2 + c]);
#pragma unroll
        for (int j = 1; j < kSub; ++j) x = fmaxf(x, fmaxf(s[j][n][c], s[j][n][2 + c]));
        mx[n][c] = x * zs[n][c];
        need = need || mx[n][c] > m_used[n][c] + kGap;
      }
    const bool moved = __any_sync(0xffffffffu, need);
    if (moved) {
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float x = mx[n][c];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
          if (x > m_used[n][c] + kGap) {
            const float to = x - kLift, al = exp2_fast(m_used[n][c] - to);   // (the first time: 0)
            m_used[n][c] = to;
            if constexpr (kE4M3) w_max[n][c] *= al;
            l_run[n][c] *= al;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
              o[n][i][c] *= al;
              o[n][i][2 + c] *= al;
            }
          }
        }
    }
    float e[kSub][kTiles][4];
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      // (a head whose scores are all -inf so far has no reference: its weights are 0)
      const float ref[2] = {m_used[n][0] > -INFINITY ? m_used[n][0] : 0.f, m_used[n][1] > -INFINITY ? m_used[n][1] : 0.f};
#pragma unroll
      for (int j = 0; j < kSub; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          e[j][n][x] = exp2_fast(fmaf(s[j][n][x], zs[n][x & 1], -ref[x & 1]));
          l_run[n][x & 1] += e[j][n][x];
        }
    }
    arrived();
    uint8_t* const vp = ring + slot * S::kBytes;
    if constexpr (kE4M3) {
      const float* sc = scales + slot * (S::kScales / 4) + ((strip * R + g4) << heads_shift) + head_l;
#pragma unroll
      for (int j = 0; j < kSub; ++j)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float x = sc[(16 * j + 8 * r) << heads_shift];
          if (partial && !cur.st.seen(s0 + 16 * j + 8 * r + g4)) x = 0.f;   // (there may be anything)
#pragma unroll
          for (int n = 0; n < kTiles; ++n) {
            e[j][n][2 * r] *= x;
            e[j][n][2 * r + 1] *= x;
          }
        }
      float top[kTiles][2];
      bool grown = moved;
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          top[n][c] = fmaxf(fabsf(e[0][n][c]), fabsf(e[0][n][2 + c]));
#pragma unroll
          for (int j = 1; j < kSub; ++j) top[n][c] = fmaxf(top[n][c], fmaxf(fabsf(e[j][n][c]), fabsf(e[j][n][2 + c])));
          grown = grown || top[n][c] * w_up[n][c] > 32768.f;
        }
      if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float x = top[n][c];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
            w_max[n][c] = fmaxf(w_max[n][c], x);
            const float up = up_of(w_max[n][c]);
            // up / w_up, both powers of two (where that is out of range the output is 0 beside what comes)
            const int k = 127 + static_cast<int>(__float_as_uint(up) >> 23) - static_cast<int>(__float_as_uint(w_up[n][c]) >> 23);
            const float by = __uint_as_float(static_cast<uint32_t>(min(max(k, 0), 254)) << 23);
            w_up[n][c] = up;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
              o[n][i][c] *= by;
              o[n][i][2 + c] *= by;
            }
          }
      }
#pragma unroll
      for (int j = 0; j < kSub; ++j)
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x) e[j][n][x] *= w_up[n][x & 1];
    }
    uint32_t wt[kSub][kTiles][2];   // weights in 16 bits; their sum is that of the unrounded ones
#pragma unroll
    for (int j = 0; j < kSub; ++j)
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int r = 0; r < 2; ++r)
          wt[j][n][r] = transposed(k16 ? pack_f16(e[j][n][2 * r], e[j][n][2 * r + 1]) : pack_bf16(e[j][n][2 * r], e[j][n][2 * r + 1]));
    if (partial) {   // rows that nobody sees may hold anything, and 0 x NaN is NaN
      constexpr int kUnits = S::kRowBytes / 16, kUnitsOf = S::kBlockBytes / 16;
      for (int i = lane; i < R * kUnits; i += 32) {
        const int r = i / kUnits, u = i % kUnits;   // (all units of a row: their order does not matter)
        if (!cur.st.seen(s0 + r)) *reinterpret_cast<uint4*>(vp + strip_at(r) + (u / kUnitsOf) * block_stride + (u % kUnitsOf) * 16) = make_uint4(0u, 0u, 0u, 0u);
      }
      tc::fence_proxy_async();   // (the next copy into the slot comes through the async proxy)
      __syncwarp();
    }
    const uint32_t vb = smem_u32(vp);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      if constexpr (!kE4M3) {
#pragma unroll
        for (int j = 0; j < kSub; ++j) {
          uint32_t w[4];
          ldmatrix_x4_trans(w, (vb + v_off[j] + (i >> 2) * block_stride) ^ ((i & 3) * 32));
#pragma unroll
          for (int n = 0; n < kTiles; ++n) mma<k16>(o[n][i], w, wt[j][n][0], wt[j][n][1]);
        }
      } else {
        // a word: dims 2 g4, 2 g4 + 1 of keys 2 t and 2 t + 1; the even dims are the tile's rows 0-7, the odd ones rows 8-15
        uint32_t c[4];
        ldmatrix_x4_trans(c, (vb + v_off[0]) ^ (i * 16));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t w[4] = {e4m3x2_to_f16x2(static_cast<uint16_t>(__byte_perm(c[2 * j], 0, 0x4420))),
                                 e4m3x2_to_f16x2(static_cast<uint16_t>(__byte_perm(c[2 * j], 0, 0x4431))),
                                 e4m3x2_to_f16x2(static_cast<uint16_t>(__byte_perm(c[2 * j + 1], 0, 0x4420))),
                                 e4m3x2_to_f16x2(static_cast<uint16_t>(__byte_perm(c[2 * j + 1], 0, 0x4431)))};
#pragma unroll
          for (int n = 0; n < kTiles; ++n) mma<k16>(o[n][i], w, wt[j][n][0], wt[j][n][1]);
        }
      }
    }
    release();
  };

  // ---- end of a (sequence, block) for this unit: the strips' parts are put together, 32 dims at a time
  const int64_t slot0 = 2 * static_cast<int64_t>(blockIdx.x);
  const int n_rows = group << heads_shift;
  const int group_inv = 65536 / group + 1;   // (row * group_inv) >> 16 is row / group for rows below 128
  auto finish = [&](bool from_start, bool to_end, bool first) {
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l_run[n][c] += __shfl_xor_sync(0xffffffffu, l_run[n][c], d);
        if (g4 == 0) ml[warp * kHeadsOf + 8 * n + 2 * t4 + c] = make_float2(m_used[n][c], l_run[n][c]);
      }
    workers_sync();
    float f[kTiles][2], down[kTiles][2];
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        down[n][c] = kE4M3 ? __uint_as_float((254u << 23) - __float_as_uint(w_up[n][c])) : 1.f;   // 1 / w_up
        const int row = 8 * n + 2 * t4 + c;
        // (each of the eight lanes of a head looks at one strip)
        const float2 mine = g4 < n_strips ? ml[((head_l << strip_shift) + g4) * kHeadsOf + row] : make_float2(-INFINITY, 0.f);
        float m = mine.x;
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        const float ref = m > -INFINITY ? m : 0.f;
        float l = mine.y * exp2_fast(mine.x - ref);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
        const bool some = l > 0.f || l != l;
        f[n][c] = some ? exp2_fast(m_used[n][c] - ref) / l : 0.f;
        if (strip == 0 && g4 == 0 && row < group) {
          const float lse2 = some ? m + log2f(l) : -INFINITY;
          if (from_start && to_end) {
            if (p.lse != nullptr) p.lse[static_cast<int64_t>(cur.b) * p.H + ((cur.block << heads_shift) + head_l) * group + row] = lse2 / paged::kLog2e;
          } else {
            p.part_lse[(slot0 + (first ? 0 : 1)) * n_rows + head_l * group + row] = lse2;
          }
        }
      }
    // With one strip a tile a warp has all of its head: it turns its rows by itself.
    const bool alone = n_strips == 1;
    auto meet = [&]() {
      if (alone) __syncwarp();
      else workers_sync();
    };
    const int i0 = alone ? lane : tid, step = alone ? 32 : 32 * kWarps, base_row = alone ? head_l * group : 0, my_rows = alone ? group : n_rows;
#pragma unroll
    for (int chunk = 0; chunk < D / S::kMergeDims; ++chunk) {
      float* mine = merge + warp * kHeadsOf * S::kMergePitch;
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int i = 0; i < S::kMergeDims / 16; ++i)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int dim = kE4M3 ? 16 * i + 2 * g4 + (x >> 1) : 16 * i + g4 + 8 * (x >> 1);
            mine[(8 * n + 2 * t4 + (x & 1)) * S::kMergePitch + dim] = o[n][S::kMergeDims / 16 * chunk + i][x] * f[n][x & 1] * down[n][x & 1];
          }
      meet();
      constexpr int kPairs = S::kMergeDims / 2;
      for (int i = i0; i < my_rows * kPairs; i += step) {   // two dims of a head
        const int rr = base_row + i / kPairs, d2 = 2 * (i % kPairs), hl = (rr * group_inv) >> 16, row = rr - hl * group;
        const float* src = merge + ((hl << strip_shift) * kHeadsOf + row) * S::kMergePitch + d2;
        float2 sum = *reinterpret_cast<const float2*>(src);
        if (!alone) {
          float2 part[kWarps - 1];
#pragma unroll
          for (int w = 1; w < kWarps; ++w)
            part[w - 1] = w < n_strips ? *reinterpret_cast<const float2*>(src + w * kHeadsOf * S::kMergePitch) : make_float2(0.f, 0.f);
#pragma unroll
          for (int w = 1; w < kWarps; ++w) {
            sum.x += part[w - 1].x;
            sum.y += part[w - 1].y;
          }
        }
        if (from_start && to_end) {
          const int h = (cur.block << heads_shift) * group + rr;
          uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<T*>(p.out) + cur.b * p.ld_out + static_cast<int64_t>(h) * D + S::kMergeDims * chunk + d2);
          *out = kF16 ? pack_f16(sum.x, sum.y) : pack_bf16(sum.x, sum.y);
        } else {
          *reinterpret_cast<float2*>(p.part_out + ((slot0 + (first ? 0 : 1)) * n_rows + rr) * D + S::kMergeDims * chunk + d2) = sum;
        }
      }
      meet();
    }
  };

  // sequences without tokens belong to no tile: their results, while the first tile is on its way
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
    if (paged::seq_length(p, b, tid == 0) > 0) continue;
    uint4* out = reinterpret_cast<uint4*>(static_cast<T*>(p.out) + b * p.ld_out);
    for (int i = tid; i < p.H * D / 8; i += 32 * kWarps) out[i] = make_uint4(0u, 0u, 0u, 0u);
    for (int i = tid; i < p.H && p.lse != nullptr; i += 32 * kWarps) p.lse[static_cast<int64_t>(b) * p.H + i] = -INFINITY;
  }
  bool from_start = cur.tile == 0, first = true;
  if (cur.left > 0) begin();
  while (cur.left > 0) {
    work();
    const bool last_of_seq = cur.tile + 1 == cur.st.count;
    if (!last_of_seq && cur.left > 1) {
      ++cur.tile;
      --cur.left;
      continue;
    }
    if (cur.left == 1 && tid == 0) paged::say_parts(p, blockIdx.x, cur, from_start, first);
    finish(from_start, last_of_seq, first);
    first = false;
    from_start = true;
    paged::advance(p, cur, shift, blocks);
    if (cur.left > 0) begin();
  }
}

// ---- parts of a sequence that several units worked on -------------------------------------------------
// Weights 2^(lse_i - max) / sum over the parts, a fixed order of addition.  A warp joins a row of few parts, or 32 dims of a row of some;
// the warps of a block share 32 dims of a row of many (a long sequence on its own is a part in every unit, and all SMs have to
// fetch them together).  Attention with it, 32 query and 8 KV heads: 64 sequences of 600 tokens, two or three parts each, 35.4 us, as some
// parts 38.7; 16 of 1500, ten parts, 26.7, as many 35.5; one of 16000, 148 parts, 19.2.
constexpr int kJoinWarps = 8, kFewParts = 8, kSomeParts = 32, kManyDims = 32;
template <typename T>
__device__ __forceinline__ void store4(T* out, const float4& x) {
  uint2 w;
  if constexpr (__is_same(T, __nv_bfloat16)) w = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
  else w = make_uint2(pack_f16(x.x, x.y), pack_f16(x.z, x.w));
  *reinterpret_cast<uint2*>(out) = w;
}
// over lanes that differ in the bits from `from` on
__device__ __forceinline__ float lanes_max(float x, int from) {
  for (int o = from; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float lanes_sum(float x, int from) {
  for (int o = from; o < 32; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ __forceinline__ void add(float4& x, float w, const float4& y) { x.x += w * y.x; x.y += w * y.y; x.z += w * y.z; x.w += w * y.w; }

template <typename T>
__global__ void __launch_bounds__(32 * kJoinWarps) paged_join_kernel(PagedAttnArgs a, int rows) {
  static_assert(paged::kJoinThreads == 32 * kJoinWarps, "threads of a block");
  __shared__ paged::JoinList list;
  __shared__ float4 acc[kJoinWarps][8];
  __shared__ float2 stats[kJoinWarps];   // {maximum, sum} of a warp's parts
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch_dependents();
  const int chunks = a.dv / kManyDims;
  auto rounds_of = [&](int n, int) {
    return n == 0 ? 0 : n <= kFewParts ? (rows + kJoinWarps - 1) / kJoinWarps : n <= kSomeParts ? (rows * chunks + kJoinWarps - 1) / kJoinWarps : rows * chunks;
  };
  int4 mine;
  int begins, owners;
  const int total = paged::join_list(a, list, tid, &mine, &begins, &owners, rounds_of);
  for (int it = blockIdx.x; it < total; it += gridDim.x) {   // block-uniform
    paged::join_find(list, tid, it, mine, begins, owners, rounds_of);
    const int4 own = list.own;
    const int n = own.x, round = list.round, unit = list.unit;
    auto slot = [&](int i) -> int64_t { return i == 0 ? own.w : 2 * (unit + i); };
    // (parts are asked for before their weights are known: one trip to L2)
    if (n <= kFewParts) {
      const int row = round * kJoinWarps + warp, d = 4 * lane;
      if (row < rows) {   // whole warps; a row has 64 or 128 dims
        float4 y[kFewParts];
#pragma unroll
        for (int i = 0; i < kFewParts; ++i)
          if (i < n && d < a.dv) y[i] = __ldcg(reinterpret_cast<const float4*>(a.part_out + (slot(i) * rows + row) * a.dv + d));
        const float lse = lane < n ? __ldcg(a.part_lse + slot(lane) * rows + row) : -INFINITY;
        const float m = lanes_max(lse, 1);
        float w = exp2f(lse - (m > -INFINITY ? m : 0.f));
        const float den = lanes_sum(w, 1);
        const bool some = den > 0.f || den != den;
        w *= some ? 1.f / den : 0.f;
        const int h = own.z * rows + row;
        if (lane == 0 && a.lse != nullptr) a.lse[static_cast<int64_t>(own.y) * a.H + h] = some ? (m + log2f(den)) / paged::kLog2e : -INFINITY;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kFewParts; ++i) {
          const float wi = __shfl_sync(0xffffffffu, w, i);
          if (i < n && d < a.dv) add(x, wi, y[i]);
        }
        if (d < a.dv) store4(static_cast<T*>(a.out) + own.y * a.ld_out + static_cast<int64_t>(h) * a.dv + d, x);
      }
    } else {
      // Eight lanes a part, four parts a warp at a time: parts first + lane / 8, `apart` further, ...
      const bool own_warp = n <= kSomeParts;
      const int piece = own_warp ? round * kJoinWarps + warp : round;
      const int row = piece / chunks, d0 = (piece - row * chunks) * kManyDims, h = own.z * rows + row, c = lane & 7;
      auto gather = [&](auto mine_c, int first, int apart, float4* sum, float* top, float* den) {   // of the warp's parts, relative to their maximum
        constexpr int kMine = decltype(mine_c)::value;
        const float* src = a.part_out + static_cast<int64_t>(row) * a.dv + d0 + 4 * c;
        float4 y[kMine];
        float w[kMine], m = -INFINITY, all = 0.f;
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
          const int i = apart * k + first + (lane >> 3);
          w[k] = -INFINITY;
          y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (i < n) {
            w[k] = __ldcg(a.part_lse + slot(i) * rows + row);
            y[k] = __ldcg(reinterpret_cast<const float4*>(src + slot(i) * rows * a.dv));
          }
          m = fmaxf(m, w[k]);
        }
        m = lanes_max(m, 8);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
          w[k] = exp2f(w[k] - (m > -INFINITY ? m : 0.f));
          all += w[k];
          add(x, w[k], y[k]);
        }
        *top = m;
        *den = lanes_sum(all, 8);
        *sum = make_float4(lanes_sum(x.x, 8), lanes_sum(x.y, 8), lanes_sum(x.z, 8), lanes_sum(x.w, 8));
      };
      auto write = [&](const float4& x, float top, float den) {   // the sum, undivided, by eight lanes
        const bool some = den > 0.f || den != den;
        const float inv = some ? 1.f / den : 0.f;
        if (lane < 8)
          store4(static_cast<T*>(a.out) + own.y * a.ld_out + static_cast<int64_t>(h) * a.dv + d0 + 4 * lane,
                 make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv));
        if (lane == 0 && d0 == 0 && a.lse != nullptr)
          a.lse[static_cast<int64_t>(own.y) * a.H + h] = some ? (top + log2f(den)) / paged::kLog2e : -INFINITY;
      };
      float4 x;
      float m, den;
      if (own_warp) {
        if (row < rows) {   // whole warps
          gather(IntC<kSomeParts / 4>{}, 0, 4, &x, &m, &den);
          write(x, m, den);
        }
      } else {
        gather(IntC<(kMaxPagedUnits + 4 * kJoinWarps - 1) / (4 * kJoinWarps)>{}, 4 * warp, 4 * kJoinWarps, &x, &m, &den);
        if (lane < 8) acc[warp][lane] = x;
        if (lane == 0) stats[warp] = make_float2(m, den);
        __syncthreads();
        if (warp == 0) {
          const float2 s = stats[lane & 7];
          float top = s.x;
          for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          const float f = exp2f(s.x - (top > -INFINITY ? top : 0.f));
          float all = f * s.y;
          for (int o = 1; o < 8; o <<= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
          x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int i = 0; i < kJoinWarps; ++i) add(x, __shfl_sync(0xffffffffu, f, i), acc[i][c]);
          write(x, top, all);
        }
      }
    }
  }
}

int heads_shift_of(int G) { return G % 8 == 0 ? 3 : G % 4 == 0 ? 2 : G % 2 == 0 ? 1 : 0; }

cudaError_t launch_paged_join(const PagedAttnArgs& a, int blocks, cudaStream_t st, int64_t* n_launch) {
  auto kernel = a.fp16 ? paged_join_kernel<__half> : paged_join_kernel<__nv_bfloat16>;
  cudaError_t e = launch_pdl(kernel, dim3(4 * a.units), dim3(32 * kJoinWarps), 0, st, a, a.H / blocks);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e == cudaSuccess) ++*n_launch;
  return e;
}

template <typename T, int D, bool kE4M3, int kTiles>
cudaError_t launch_t(const PagedAttnArgs& a, cudaStream_t st, int64_t* n_launch) {
  using S = Shape<D, kE4M3, kTiles>;
  static_assert(S::kSmem <= 227 * 1024, "shared memory of a block");
  const uint64_t rows = static_cast<uint64_t>(a.n_pages > 0 ? a.n_pages : 1) << a.page_shift;
  const int hs = heads_shift_of(a.G), tile_keys = S::kRows << (3 - hs);
  const uint32_t box_rows = (1 << a.page_shift) < tile_keys ? 1 << a.page_shift : tile_keys;
  CUtensorMap k_map, v_map;
  const bool ok = kE4M3 ? make_map_u8_blocks(&k_map, a.k_pool, D, a.G, rows, a.ld_k, box_rows, 1 << hs) && make_map_u8_blocks(&v_map, a.v_pool, D, a.G, rows, a.ld_v, box_rows, 1 << hs)
                        : make_map_16bit_blocks(&k_map, a.k_pool, a.G * D / 64, rows, a.ld_k, box_rows, S::kBlocks << hs) &&
                              make_map_16bit_blocks(&v_map, a.v_pool, a.G * D / 64, rows, a.ld_v, box_rows, S::kBlocks << hs);
  if (!ok) return cudaErrorInvalidValue;
  auto kernel = paged_attn_kernel<T, D, kE4M3, kTiles>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3(a.units), dim3(kThreads), S::kSmem, st, k_map, v_map, a, hs);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ++*n_launch;
  return launch_paged_join(a, a.G >> hs, st, n_launch);
}
template <typename T, int D, bool kE4M3>
cudaError_t launch_n(const PagedAttnArgs& a, cudaStream_t st, int64_t* n_launch) {
  return a.H / a.G <= 8 ? launch_t<T, D, kE4M3, 1>(a, st, n_launch) : launch_t<T, D, kE4M3, 2>(a, st, n_launch);
}
template <typename T>
cudaError_t launch_d(const PagedAttnArgs& a, cudaStream_t st, int64_t* n_launch) {
  if (a.d == 128) return a.e4m3 ? launch_n<T, 128, true>(a, st, n_launch) : launch_n<T, 128, false>(a, st, n_launch);
  return a.e4m3 ? launch_n<T, 64, true>(a, st, n_launch) : launch_n<T, 64, false>(a, st, n_launch);
}

}  // namespace

int paged_rows(int latent, int H, int G) { return latent ? 64 : (H / G) << heads_shift_of(G); }
int64_t paged_entries(int latent, int G, int64_t max_len) {
  const int hs = heads_shift_of(G), keys = latent ? 64 : 16 << (3 - hs);   // (at least so many keys a tile)
  return (max_len / keys + 2) * (G >> hs);
}

cudaError_t launch_paged_attn(const PagedAttnArgs& a, cudaStream_t st, int64_t* n_launch) {
  return a.fp16 ? launch_d<__half>(a, st, n_launch) : launch_d<__nv_bfloat16>(a, st, n_launch);
}

}  // namespace lsa
