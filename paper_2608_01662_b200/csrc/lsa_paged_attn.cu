// lsa_paged_attn for caches with separate keys and values: one query per sequence, up to 16 query heads per KV head.
//
// A query head's 64 or 128 dims meet each cached key and value once: at most 16 flop per byte read, so the kernel has to keep
// HBM busy and the products have to stay out of its way.  The query heads of a KV head are the 16 rows of m16n8k16 MMAs.  A
// warp works alone: it copies strips of 16 or 32 consecutive tokens of one KV head (4 KB of keys, 4 KB of values) into a ring of
// its own by cp.async, and keeps the running maximum, sum and output of its strips in registers, so that no warp waits for
// another until the end of a sequence.  A tile is what the eight warps of a block take in one go: all the KV heads of a block
// (up to eight; a row of the cache is then read whole) times as many strips as make up eight.
//
// e4m3 caches: a code is exact in fp16, and so is a query scaled by a power of two of its own head, so the scores' products
// are fp16 MMAs of codes and the scale of a key is applied to the score.  A value's scale is applied to its weight before that is
// rounded to bf16 (which has the range for any scale); the codes become bf16, exactly.
#include "lsa_paged.cuh"

namespace lsa {

namespace {

using paged::Cursor;
using paged::exp2_fast;
using paged::SeqTiles;

constexpr int kWarps = 8;
constexpr float kRescaleGap = 8.f;   // the output is rescaled only when a row's maximum grows by more than 2^8

template <int D, bool kE4M3>
struct Strip {
  static constexpr int kElem = kE4M3 ? 1 : 2, kRowBytes = D * kElem;
  static constexpr int kRows = 4096 / kRowBytes < 32 ? 4096 / kRowBytes : 32;
  static constexpr int kBytes = kRows * kRowBytes;                 // of keys, and of values
  static constexpr int kScaleBytes = kE4M3 ? 2 * kRows * 4 : 0;
  static constexpr int kStage = 2 * kBytes + kScaleBytes;
  static constexpr int kStages = kBytes == 4096 ? 3 : 5;
  static constexpr int kRowShift = kRows == 32 ? 5 : 4;
  static constexpr int kRing = kWarps * kStages * kStage;
  static constexpr int kMergePitch = 36;                           // floats: 32 dims of a row and a gap
  static constexpr int kMerge = kWarps * 16 * kMergePitch * 4;
  static constexpr int kSmem = kRing + kMerge + kWarps * 16 * 8;
};

// 16-byte unit u of row r of a strip: the units that one ldmatrix phase reads (eight rows) lie in different banks.
template <int kRowBytes>
__device__ __forceinline__ uint32_t unit_at(int r, int u) {
  if constexpr (kRowBytes == 64) return (r >> 1) * 128 + (((((r & 1) << 2) | u) ^ ((r >> 1) & 7)) << 4);
  else return swz<kRowBytes>(r, u);
}

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
  __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
  return static_cast<uint32_t>(h.x) | (static_cast<uint32_t>(h.y) << 16);
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, int src_bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst), "l"(src), "r"(src_bytes));
}

// heads: KV heads that a block works on at the same time (8, 4, 2 or 1, a divisor of G); strips: strips of a tile (8 / heads).
template <typename T, int D, bool kE4M3>
__global__ void __launch_bounds__(32 * kWarps, 1) paged_attn_kernel(PagedAttnArgs a, int heads_shift) {
  using S = Strip<D, kE4M3>;
  constexpr bool kF16 = sizeof(T) == 2 && !__is_same(T, __nv_bfloat16);
  constexpr int R = S::kRows, kTiles = R / 8;       // n-tiles of a strip's scores
  extern __shared__ __align__(128) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g4 = lane >> 2, t4 = lane & 3;
  const int strip_shift = 3 - heads_shift, n_strips = 1 << strip_shift;
  const int head_l = warp >> strip_shift, strip = warp & (n_strips - 1);
  const int shift = S::kRowShift + strip_shift;     // keys of a tile
  const int blocks = a.G >> heads_shift;
  const int group = a.H / a.G;
  uint8_t* const ring = smem + warp * S::kStages * S::kStage;
  float* const merge = reinterpret_cast<float*>(smem + S::kRing);
  float2* const ml = reinterpret_cast<float2*>(smem + S::kRing + S::kMerge);   // {maximum, sum} per warp and row

  pdl_wait();
  pdl_launch_dependents();

  // sequences without tokens belong to no tile
  for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
    if (paged::seq_length(a, b, tid == 0) > 0) continue;
    T* out = static_cast<T*>(a.out) + b * a.ld_out;
    for (int i = tid; i < a.H * D; i += 32 * kWarps) out[i] = T(0.f);
    for (int i = tid; i < a.H && a.lse != nullptr; i += 32 * kWarps) a.lse[static_cast<int64_t>(b) * a.H + i] = -INFINITY;
  }

  Cursor cur = paged::first_entry(a, blockIdx.x, shift, blocks, lane);
  if (cur.left == 0) {
    if (tid == 0) a.parts[blockIdx.x] = make_int4(0, 0, 0, 0);
    return;
  }
  const bool first_is_start = cur.tile == 0;   // the unit's first entry begins its (sequence, block)
  Cursor ahead = cur;
  const int page_mask = (1 << a.page_shift) - 1;

  // ---- copies: the strip at `ahead`, whose page numbers were fetched one call before
  int pages[R / 16];
  auto fetch_pages = [&]() {
    const int s0 = ahead.st.first_key(ahead.tile, shift) + strip * R;
#pragma unroll
    for (int h = 0; h < R / 16; ++h) {
      pages[h] = -1;
      if (ahead.left > 0 && ahead.st.any_seen(s0 + 16 * h, 16)) {
        const int p = a.page_table[ahead.b * a.pt_stride + ((s0 + 16 * h) >> a.page_shift)];
        if (p >= 0 && p < a.n_pages) pages[h] = p;
        else paged::report_index(a.notice);
      }
    }
  };
  auto copy = [&](int stage) {
    if (ahead.left > 0) {
      const int s0 = ahead.st.first_key(ahead.tile, shift) + strip * R;
      const int g = (ahead.block << heads_shift) + head_l;
      const uint32_t dst = smem_u32(ring + stage * S::kStage);
      const uint8_t* kp = static_cast<const uint8_t*>(a.k_pool);
      const uint8_t* vp = static_cast<const uint8_t*>(a.v_pool);
      constexpr int kUnits = S::kRowBytes / 16, kAtOnce = 32 / kUnits;   // units of a row; rows that the warp copies with one instruction
      const int u = lane % kUnits, r0 = lane / kUnits;
#pragma unroll
      for (int h = 0; h < R / 16; ++h) {
        const int64_t row0 = (static_cast<int64_t>(max(pages[h], 0)) << a.page_shift) + ((s0 + 16 * h) & page_mask);
        const uint8_t* ks = kp + (row0 + r0) * a.ld_k * S::kElem + g * S::kRowBytes + u * 16;
        const uint8_t* vs = vp + (row0 + r0) * a.ld_v * S::kElem + g * S::kRowBytes + u * 16;
#pragma unroll
        for (int i = 0; i < 16 / kAtOnce; ++i) {
          const int r = 16 * h + i * kAtOnce + r0;
          const int bytes = pages[h] >= 0 && ahead.st.seen(s0 + r) ? 16 : 0;   // what is not seen is a row of zeros
          cp_async16(dst + unit_at<S::kRowBytes>(r, u), ks + static_cast<int64_t>(i * kAtOnce) * a.ld_k * S::kElem, bytes);
          cp_async16(dst + S::kBytes + unit_at<S::kRowBytes>(r, u), vs + static_cast<int64_t>(i * kAtOnce) * a.ld_v * S::kElem, bytes);
        }
      }
      if constexpr (kE4M3) {
        static_assert(R == 32, "a lane per row of scales");
        const int p = lane < 16 ? pages[0] : pages[R / 16 - 1];
        const int64_t row = (static_cast<int64_t>(max(p, 0)) << a.page_shift) + ((s0 + lane) & page_mask);
        const int bytes = p >= 0 && ahead.st.seen(s0 + lane) ? 4 : 0;
        cp_async4(dst + 2 * S::kBytes + lane * 4, a.k_scale + row * a.G + g, bytes);
        cp_async4(dst + 2 * S::kBytes + R * 4 + lane * 4, a.v_scale + row * a.G + g, bytes);
      }
      paged::advance(a, ahead, shift, blocks);
      fetch_pages();
    }
    cp_async_commit();
  };

  // ---- the state of a (sequence, block): query fragments, output, maxima, sums
  uint32_t qf[D / 16][4];
  float zs[2];
  float o[D / 8][4];
  float m_used[2], l_run[2];
  auto begin = [&]() {
    const int head0 = ((cur.block << heads_shift) + head_l) * group;
    const T* q = static_cast<const T*>(a.q) + cur.b * a.ld_q + static_cast<int64_t>(head0) * D;
    zs[0] = zs[1] = a.scale2;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const bool on = g4 + 8 * r < group;
      const uint32_t* row = reinterpret_cast<const uint32_t*>(q + (g4 + 8 * r) * D);   // pairs of dims
      if constexpr (!kE4M3) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          qf[k][r] = on ? row[8 * k + t4] : 0u;
          qf[k][2 + r] = on ? row[8 * k + 4 + t4] : 0u;
        }
      } else {   // dims 16 k + 4 t .. + 3 take the places of the columns 2 t, 2 t + 1, 2 t + 8, 2 t + 9 of step k
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint2 w = on ? *reinterpret_cast<const uint2*>(row + 8 * k + 2 * t4) : make_uint2(0u, 0u);
          qf[k][r] = w.x;
          qf[k][2 + r] = w.y;
        }
        if constexpr (!kF16) {
          float top = 0.f;
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&qf[k][2 * h + r]));
              top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          // largest element in [2^14, 2^15): what lies 2^-29 below it still has all its bits
          const int sh = e5m2_head_shift(top);
          const float up = __uint_as_float(static_cast<uint32_t>(127 + sh) << 23);
          zs[r] *= __uint_as_float(static_cast<uint32_t>(127 - sh) << 23);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&qf[k][2 * h + r]));
              qf[k][2 * h + r] = pack_f16(f.x * up, f.y * up);
            }
        }
      }
      m_used[r] = -INFINITY;
      l_run[r] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  };

  // ---- one strip
  auto work = [&](int stage) {
    const int s0 = cur.st.first_key(cur.tile, shift) + strip * R;
    if (!cur.st.any_seen(s0, R)) return;
    const uint32_t ks = smem_u32(ring + stage * S::kStage), vs = ks + S::kBytes;
    float s[kTiles][4];
#pragma unroll
    for (int j = 0; j < kTiles; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      if constexpr (!kE4M3) {
#pragma unroll
        for (int j = 0; j < R / 16; ++j) {
          uint32_t w[4];
          ldmatrix_x4(w, ks + unit_at<S::kRowBytes>(16 * j + (lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)));
          if constexpr (kF16) {
            mma_f16(s[2 * j], qf[k], w[0], w[1]);
            mma_f16(s[2 * j + 1], qf[k], w[2], w[3]);
          } else {
            mma_bf16(s[2 * j], qf[k], w[0], w[1]);
            mma_bf16(s[2 * j + 1], qf[k], w[2], w[3]);
          }
        }
      } else {
        uint32_t w[4];   // four codes of a key: dims 16 k + 4 t .. + 3, keys 8 j + lane / 4
        ldmatrix_x4(w, ks + unit_at<S::kRowBytes>(lane, k));
#pragma unroll
        for (int j = 0; j < 4; ++j) mma_f16(s[j], qf[k], e4m3x2_to_f16x2(w[j] & 0xffffu), e4m3x2_to_f16x2(w[j] >> 16));
      }
    }
    // scores in log2 units; the thread's keys are 8 j + 2 t, + 1, its rows g4 and g4 + 8
    float2 vsc[kTiles];
    const float* sc = reinterpret_cast<const float*>(ring + stage * S::kStage + 2 * S::kBytes);
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
      float2 ksc = make_float2(1.f, 1.f);
      if constexpr (kE4M3) {
        ksc = *reinterpret_cast<const float2*>(sc + 8 * j + 2 * t4);
        vsc[j] = *reinterpret_cast<const float2*>(sc + R + 8 * j + 2 * t4);
        s[j][0] *= ksc.x; s[j][1] *= ksc.y; s[j][2] *= ksc.x; s[j][3] *= ksc.y;
      }
      s[j][0] *= zs[0]; s[j][1] *= zs[0]; s[j][2] *= zs[1]; s[j][3] *= zs[1];
    }
    if (!cur.st.all_seen(s0, R)) {
#pragma unroll
      for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          if (!cur.st.seen(s0 + 8 * j + 2 * t4 + c)) s[j][c] = s[j][2 + c] = -INFINITY;
    }
    float mx[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float x = fmaxf(s[0][2 * r], s[0][2 * r + 1]);
#pragma unroll
      for (int j = 1; j < kTiles; ++j) x = fmaxf(x, fmaxf(s[j][2 * r], s[j][2 * r + 1]));
      x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
      mx[r] = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
    }
    const bool grow0 = mx[0] > m_used[0] + kRescaleGap, grow1 = mx[1] > m_used[1] + kRescaleGap;
    if (__any_sync(0xffffffffu, grow0 || grow1)) {
      float al[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        al[r] = 1.f;
        if (r == 0 ? grow0 : grow1) {
          al[r] = exp2_fast(m_used[r] - mx[r]);   // (the first time: 0)
          m_used[r] = mx[r];
        }
        l_run[r] *= al[r];
      }
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        o[i][0] *= al[0]; o[i][1] *= al[0]; o[i][2] *= al[1]; o[i][3] *= al[1];
      }
    }
    // (a row whose scores are all -inf so far has no maximum: its weights are 0)
    const float ref[2] = {m_used[0] > -INFINITY ? m_used[0] : 0.f, m_used[1] > -INFINITY ? m_used[1] : 0.f};
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
#pragma unroll
      for (int c = 0; c < 4; ++c) s[j][c] = exp2_fast(s[j][c] - ref[c >> 1]);
      l_run[0] += s[j][0] + s[j][1];
      l_run[1] += s[j][2] + s[j][3];
      if constexpr (kE4M3) {
        s[j][0] *= vsc[j].x; s[j][1] *= vsc[j].y; s[j][2] *= vsc[j].x; s[j][3] *= vsc[j].y;
      }
    }
#pragma unroll
    for (int j = 0; j < R / 16; ++j) {
      uint32_t p[4];   // weights of keys 16 j .. + 15: rounded to 16 bits, at most 2^8, their sum kept in fp32 above
      if constexpr (kF16 && !kE4M3) {
        p[0] = pack_f16(s[2 * j][0], s[2 * j][1]); p[1] = pack_f16(s[2 * j][2], s[2 * j][3]);
        p[2] = pack_f16(s[2 * j + 1][0], s[2 * j + 1][1]); p[3] = pack_f16(s[2 * j + 1][2], s[2 * j + 1][3]);
      } else {
        p[0] = pack_bf16(s[2 * j][0], s[2 * j][1]); p[1] = pack_bf16(s[2 * j][2], s[2 * j][3]);
        p[2] = pack_bf16(s[2 * j + 1][0], s[2 * j + 1][1]); p[3] = pack_bf16(s[2 * j + 1][2], s[2 * j + 1][3]);
      }
      const int r = 16 * j + (lane & 7) + ((lane >> 3) & 1) * 8;
#pragma unroll
      for (int d = 0; d < S::kRowBytes / 32; ++d) {   // two 16-byte units of the rows
        uint32_t w[4];
        ldmatrix_x4_trans(w, vs + unit_at<S::kRowBytes>(r, 2 * d + (lane >> 4)));
        if constexpr (!kE4M3) {
          if constexpr (kF16) {
            mma_f16(o[2 * d], p, w[0], w[1]);
            mma_f16(o[2 * d + 1], p, w[2], w[3]);
          } else {
            mma_bf16(o[2 * d], p, w[0], w[1]);
            mma_bf16(o[2 * d + 1], p, w[2], w[3]);
          }
        } else {
          // a word: dims 2 n, 2 n + 1 (n = lane / 4) of keys 2 t and 2 t + 1; the even dims are one n-tile, the odd ones another
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t lo = w[2 * h], hi = w[2 * h + 1];
            mma_bf16(o[4 * d + 2 * h], p, e4m3x2_to_bf16x2(static_cast<uint16_t>(__byte_perm(lo, 0, 0x4420))),
                     e4m3x2_to_bf16x2(static_cast<uint16_t>(__byte_perm(hi, 0, 0x4420))));
            mma_bf16(o[4 * d + 2 * h + 1], p, e4m3x2_to_bf16x2(static_cast<uint16_t>(__byte_perm(lo, 0, 0x4431))),
                     e4m3x2_to_bf16x2(static_cast<uint16_t>(__byte_perm(hi, 0, 0x4431))));
          }
        }
      }
    }
  };

  // ---- end of a (sequence, block) for this unit: the strips' parts are put together, 32 dims at a time
  const int64_t slot0 = 2 * static_cast<int64_t>(blockIdx.x);
  auto finish = [&](bool from_start, bool to_end, bool first) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l_run[r] += __shfl_xor_sync(0xffffffffu, l_run[r], 1);
      l_run[r] += __shfl_xor_sync(0xffffffffu, l_run[r], 2);
      if (t4 == 0) ml[warp * 16 + g4 + 8 * r] = make_float2(m_used[r], l_run[r]);
    }
    __syncthreads();
    float f[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float m = -INFINITY, l = 0.f;
      const float2* all = ml + (head_l << strip_shift) * 16 + g4 + 8 * r;
      for (int w = 0; w < n_strips; ++w) m = fmaxf(m, all[16 * w].x);
      const float ref = m > -INFINITY ? m : 0.f;
      for (int w = 0; w < n_strips; ++w) l += all[16 * w].y * exp2_fast(all[16 * w].x - ref);
      f[r] = l > 0.f || l != l ? exp2_fast(m_used[r] - ref) / l : 0.f;
      const int row = g4 + 8 * r, h = ((cur.block << heads_shift) + head_l) * group + row;
      if (strip == 0 && t4 == 0 && row < group) {
        const float lse2 = l > 0.f || l != l ? m + log2f(l) : -INFINITY;
        if (from_start && to_end) {
          if (a.lse != nullptr) a.lse[static_cast<int64_t>(cur.b) * a.H + h] = lse2 / paged::kLog2e;
        } else {
          a.part_lse[(slot0 + (first ? 0 : 1)) * (group << heads_shift) + head_l * group + row] = lse2;
        }
      }
    }
    const int rows = group << heads_shift;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      float* mine = merge + warp * 16 * S::kMergePitch;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int x = 0; x < 4; ++x) {   // (e4m3: the n-tiles of a unit are its even and its odd dims)
          const int col = 2 * t4 + (x & 1);
          const int dim = kE4M3 ? 16 * (i >> 1) + 2 * col + (i & 1) : 8 * i + col;
          mine[(g4 + 8 * (x >> 1)) * S::kMergePitch + dim] = o[4 * c + i][x] * f[x >> 1];
        }
      __syncthreads();
      for (int i = tid; i < rows * 16; i += 32 * kWarps) {   // two dims of a row
        const int rr = i >> 4, d2 = 2 * (i & 15), hl = rr / group, row = rr - hl * group;
        float2 sum = make_float2(0.f, 0.f);
        for (int w = 0; w < n_strips; ++w) {
          const float2 x = *reinterpret_cast<const float2*>(merge + (((hl << strip_shift) + w) * 16 + row) * S::kMergePitch + d2);
          sum.x += x.x;
          sum.y += x.y;
        }
        const int h = ((cur.block << heads_shift) + hl) * group + row;
        if (from_start && to_end) {
          uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + cur.b * a.ld_out + static_cast<int64_t>(h) * D + 32 * c + d2);
          *out = kF16 ? pack_f16(sum.x, sum.y) : pack_bf16(sum.x, sum.y);
        } else {
          *reinterpret_cast<float2*>(a.part_out + ((slot0 + (first ? 0 : 1)) * rows + rr) * D + 32 * c + d2) = sum;
        }
      }
      __syncthreads();
    }
  };

  fetch_pages();
#pragma unroll
  for (int i = 0; i < S::kStages - 1; ++i) copy(i);
  begin();
  bool from_start = first_is_start, first = true;
  int stage = 0;
  while (true) {
    cp_async_wait<S::kStages - 2>();
    __syncwarp();
    work(stage);
    __syncwarp();
    copy(stage == 0 ? S::kStages - 1 : stage - 1);   // the stage of the strip before
    stage = stage == S::kStages - 1 ? 0 : stage + 1;
    const bool last_of_seq = cur.tile + 1 == cur.st.count;
    if (cur.left == 1 && tid == 0) paged::say_parts(a, blockIdx.x, cur, from_start, first);
    if (last_of_seq || cur.left == 1) {
      finish(from_start, last_of_seq, first);
      first = false;
    }
    const bool more = cur.left > 1;
    const bool other = paged::advance(a, cur, shift, blocks);
    if (!more) break;
    if (other) {
      begin();
      from_start = true;
    }
  }
  cp_async_wait<0>();
}

// ---- parts of a sequence that several units worked on -------------------------------------------------
// Weights 2^(lse_i - max) / sum over the parts, added in the parts' order.  A warp joins a row of few parts; the warps of a block share
// 128 dims of a row of many (one long sequence is 148 parts: 300 KB of a latent row).
constexpr int kJoinWarps = 8, kFewParts = 8, kManyDims = 128;
template <typename T>
__device__ __forceinline__ void store4(T* out, const float4& x) {
  uint2 w;
  if constexpr (__is_same(T, __nv_bfloat16)) w = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
  else w = make_uint2(pack_f16(x.x, x.y), pack_f16(x.z, x.w));
  *reinterpret_cast<uint2*>(out) = w;
}
template <typename T>
__global__ void __launch_bounds__(32 * kJoinWarps) paged_join_kernel(PagedAttnArgs a, int rows) {
  __shared__ int4 parts[kMaxPagedUnits];
  __shared__ int upto[kMaxPagedUnits];     // rounds of a block for the owners up to this one
  __shared__ float4 acc[kJoinWarps][32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch_dependents();
  for (int i = tid; i < a.units; i += 32 * kJoinWarps) parts[i] = __ldcg(a.parts + i);
  // (units that gave up on a wait have left nothing, and nothing said about it)
  if (__syncthreads_or(a.status != nullptr && *reinterpret_cast<const volatile int*>(a.status) != 0)) return;
  const int chunks = max(a.dv / kManyDims, 1), chunk_dims = min(a.dv, kManyDims);
  auto rounds = [&](int n) { return n == 0 ? 0 : n <= kFewParts ? (rows + kJoinWarps - 1) / kJoinWarps : rows * chunks; };
  if (warp == 0) {
    int sum = 0;
    for (int i0 = 0; i0 < a.units; i0 += 32) {
      int x = i0 + lane < a.units ? rounds(parts[i0 + lane].x) : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (i0 + lane < a.units) upto[i0 + lane] = sum + x;
      sum += __shfl_sync(0xffffffffu, x, 31);
    }
  }
  __syncthreads();
  const int total = upto[a.units - 1];
  for (int it = blockIdx.x; it < total; it += gridDim.x) {   // block-uniform
    int lo = 0, hi = a.units - 1;   // the first owner with upto > it
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (upto[mid] > it) hi = mid;
      else lo = mid + 1;
    }
    const int4 own = parts[lo];
    const int n = own.x, round = it - (lo > 0 ? upto[lo - 1] : 0);
    auto slot = [&](int i) -> int64_t { return i == 0 ? own.w : 2 * (lo + i); };
    // the weights of the parts of a row, a lane's being those of parts lane, lane + 32, ...
    constexpr int kMine = (kMaxPagedUnits + 31) / 32;
    auto weights = [&](int row, float (&w)[kMine], float* lse) {
      float m = -INFINITY;
#pragma unroll
      for (int k = 0; k < kMine; ++k) {
        w[k] = 32 * k + lane < n ? __ldcg(a.part_lse + slot(32 * k + lane) * rows + row) : -INFINITY;
        m = fmaxf(m, w[k]);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      const float ref = m > -INFINITY ? m : 0.f;
      float den = 0.f;
#pragma unroll
      for (int k = 0; k < kMine; ++k) {
        w[k] = exp2f(w[k] - ref);
        den += w[k];
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
      const bool some = den > 0.f || den != den;
      const float inv = some ? 1.f / den : 0.f;
#pragma unroll
      for (int k = 0; k < kMine; ++k) w[k] *= inv;
      *lse = some ? (m + log2f(den)) / paged::kLog2e : -INFINITY;
    };
    float w[kMine], lse;
    if (n <= kFewParts) {
      const int row = round * kJoinWarps + warp;
      if (row < rows) {   // whole warps
        weights(row, w, &lse);
        const int h = own.z * rows + row;
        if (lane == 0 && a.lse != nullptr) a.lse[static_cast<int64_t>(own.y) * a.H + h] = lse;
        for (int d = 4 * lane; d < a.dv; d += 128) {
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int i = 0; i < kFewParts; ++i) {
            if (i < n) {
              const float4 y = __ldcg(reinterpret_cast<const float4*>(a.part_out + (slot(i) * rows + row) * a.dv + d));
              const float wi = __shfl_sync(__activemask(), w[0], i);
              x.x += wi * y.x; x.y += wi * y.y; x.z += wi * y.z; x.w += wi * y.w;
            }
          }
          store4(static_cast<T*>(a.out) + own.y * a.ld_out + static_cast<int64_t>(h) * a.dv + d, x);
        }
      }
    } else {
      const int row = round / chunks, d0 = (round - row * chunks) * chunk_dims;
      const int h = own.z * rows + row;
      weights(row, w, &lse);
      if (tid == 0 && d0 == 0 && a.lse != nullptr) a.lse[static_cast<int64_t>(own.y) * a.H + h] = lse;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      const bool on = 4 * lane < chunk_dims;
      const float* src = a.part_out + static_cast<int64_t>(row) * a.dv + d0 + (on ? 4 * lane : 0);
#pragma unroll
      for (int k = 0; k < kMine; ++k) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {   // parts 32 k + 8 j + warp
          const int i = 32 * k + 8 * j + warp;
          const float wi = __shfl_sync(0xffffffffu, w[k], 8 * j + warp);
          if (i < n) {
            const float4 y = __ldcg(reinterpret_cast<const float4*>(src + slot(i) * rows * a.dv));
            x.x += wi * y.x; x.y += wi * y.y; x.z += wi * y.z; x.w += wi * y.w;
          }
        }
      }
      __syncthreads();   // (the round before has been read)
      acc[warp][lane] = x;
      __syncthreads();
      if (warp == 0) {
#pragma unroll
        for (int i = 1; i < kJoinWarps; ++i) {
          const float4 y = acc[i][lane];
          x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
        }
        if (on) store4(static_cast<T*>(a.out) + own.y * a.ld_out + static_cast<int64_t>(h) * a.dv + d0 + 4 * lane, x);
      }
    }
  }
}

int heads_shift_of(int G) { return G % 8 == 0 ? 3 : G % 4 == 0 ? 2 : G % 2 == 0 ? 1 : 0; }

static cudaError_t launch_paged_join(const PagedAttnArgs& a, int blocks, cudaStream_t st, int64_t* n_launch) {
  auto kernel = a.fp16 ? paged_join_kernel<__half> : paged_join_kernel<__nv_bfloat16>;
  cudaError_t e = launch_pdl(kernel, dim3(4 * a.units), dim3(32 * kJoinWarps), 0, st, a, a.H / blocks);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e == cudaSuccess) ++*n_launch;
  return e;
}

template <typename T, int D, bool kE4M3>
cudaError_t launch_t(const PagedAttnArgs& a, cudaStream_t st, int64_t* n_launch) {
  using S = Strip<D, kE4M3>;
  static_assert(S::kSmem <= 227 * 1024, "shared memory of a block");
  auto kernel = paged_attn_kernel<T, D, kE4M3>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
  if (e != cudaSuccess) return e;
  const int hs = heads_shift_of(a.G);
  e = launch_pdl(kernel, dim3(a.units), dim3(32 * kWarps), S::kSmem, st, a, hs);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ++*n_launch;
  return launch_paged_join(a, a.G >> hs, st, n_launch);
}
template <typename T>
cudaError_t launch_d(const PagedAttnArgs& a, cudaStream_t st, int64_t* n_launch) {
  if (a.d == 128) return a.e4m3 ? launch_t<T, 128, true>(a, st, n_launch) : launch_t<T, 128, false>(a, st, n_launch);
  return a.e4m3 ? launch_t<T, 64, true>(a, st, n_launch) : launch_t<T, 64, false>(a, st, n_launch);
}

}  // namespace

int paged_rows(int latent, int H, int G) { return latent ? 64 : (H / G) << heads_shift_of(G); }
int64_t paged_entries(const PagedAttnArgs& a) {
  const int hs = heads_shift_of(a.G), keys = a.latent ? 64 : 16 << (3 - hs);   // (at least so many keys a tile)
  return static_cast<int64_t>(a.batch) * (a.max_len / keys + 2) * (a.G >> hs);
}


cudaError_t launch_paged_attn(const PagedAttnArgs& a, cudaStream_t st, int64_t* n_launch) {
  return a.fp16 ? launch_d<__half>(a, st, n_launch) : launch_d<__nv_bfloat16>(a, st, n_launch);
}

}  // namespace lsa
