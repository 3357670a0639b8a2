// lsa_paged_attn over latent rows (absorbed MLA: up to 64 query heads, d_qk = 576, the value is the first 512 dims of the key
// row) on the 5th-generation tensor cores.
//
// A token's 1152 bytes meet 64 heads: 121 flop per byte, so HBM is the bound only as long as the products run on tcgen05 and
// the softmax stays beside them.  The 64 heads are the M = 64 rows of every MMA (rows of absent heads are zero).  A unit of the
// grid works through its share of the list of 64-token tiles (lsa_paged.cuh), one (sequence) after another:
//
//   warp 4      copies: a tile lies inside one cache page, so it is one TMA box (nine column blocks of 64 rows x 128 bytes,
//               128B-swizzled), into a ring of three.  Every tile is 73.7 KB: while one is worked on two are on their way.
//   warp 5      S = Q K^T, M64 N64 K16, Q in tensor memory (its last 64 dims in shared memory), as two accumulation chains
//               in the two halves of the lanes (an M = 64 accumulator uses 16 lanes of each 32); two S buffers.
//   warps 0-3   softmax: the two partial sums are added, running maximum with lazy rescaling of O, exp2, fp32 row sums, P in
//               16 bits into the tile's last column block, which only Q K^T reads.  At a sequence's end they fetch the next Q and
//               write O.  Rows of a tile that nobody sees are zeroed there before they become values: 0 x NaN is NaN.
//   warp 6      O += P V, tcgen05.mma.ws M64 N256 K16; V is the tile read MN-major, so a row is fetched once.
//
// Tensor memory columns:   0-255  O: value dims 0-255 in columns 0-127, 256-511 in 128-255; lanes 0-63 hold the first 128
//                                 dims of each, lanes 64-127 the second, lane l (mod 64) = head l
//                        256-383  Q[:, 0:512], two dims a column, dims 0-255 in lanes 0-15 of each 32, 256-511 in 16-31
//                        384-511  S, two buffers: the first chain's partial sum in lanes 0-15 of each 32, the second's in 16-31
#include "lsa_paged.cuh"
#include "lsa_tc.cuh"

namespace lsa {

namespace {

using paged::Cursor;
using paged::exp2_fast;

constexpr int kHeads = 64, kDQK = 576, kDV = 512;
constexpr int kShift = 6, kTileKeys = 1 << kShift;
constexpr int kAtoms = kDQK / 64;
constexpr int kAtomBytes = kTileKeys * 128;
constexpr int kSlotBytes = kAtoms * kAtomBytes;
constexpr int kRing = 3;
constexpr int kSoftmaxWarps = 4, kCopyWarp = 4, kQkWarp = 5, kPvWarp = 6, kThreads = 224;
constexpr int kSoftmaxThreads = 32 * kSoftmaxWarps;
constexpr uint32_t kTmemCols = 512, kColQ = 256, kColS = 384, kSBuf = 64;
constexpr float kRescaleGap = 8.f;   // O is rescaled only when a row's maximum grows by more than 2^8

struct LatentSmem {
  alignas(1024) uint8_t k[kRing][kAtoms][kAtomBytes];
  alignas(1024) uint8_t q_rope[kAtomBytes];
  alignas(8) uint64_t k_full[kRing], k_empty[kRing], p_ready[kRing], pv_done[kRing], s_full[2], s_free[2], q_ready;
  uint32_t tmem_slot;
  float factor[kHeads];   // of a rescaling of O; at a sequence's end 1 / l
};

__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxThreads) : "memory"); }
__device__ __forceinline__ bool softmax_any(bool v) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred a, b;\n\tsetp.ne.b32 a, %1, 0;\n\tbar.red.or.pred b, 1, %2, a;\n\tselp.b32 %0, 1, 0, b;\n\t}"
               : "=r"(r) : "r"(static_cast<uint32_t>(v)), "n"(kSoftmaxThreads) : "memory");
  return r != 0;
}
__device__ __forceinline__ void stmatrix_x4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
template <bool kF16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if constexpr (kF16) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    return pack_bf16(x, y);
  }
}
// (both operands of an MMA have the one type)
template <bool kF16>
__host__ __device__ constexpr uint32_t idesc_16(int M, int N, int a_mn, int b_mn) {
  return kF16 ? tc::idesc_bf16(M, N, a_mn, b_mn) & ~((1u << 7) | (1u << 10)) : tc::idesc_bf16(M, N, a_mn, b_mn);
}

template <bool kF16>
__global__ void __launch_bounds__(kThreads, 1) paged_latent_kernel(const __grid_constant__ CUtensorMap k_map, PagedAttnArgs a) {
  extern __shared__ uint8_t smem_raw[];
  LatentSmem& sm = *reinterpret_cast<LatentSmem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);

  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) {
      tc::mbar_init(smem_u32(&sm.k_full[i]), 1);
      tc::mbar_init(smem_u32(&sm.k_empty[i]), 1);
      tc::mbar_init(smem_u32(&sm.p_ready[i]), 1);
      tc::mbar_init(smem_u32(&sm.pv_done[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(smem_u32(&sm.s_full[i]), 1);
      tc::mbar_init(smem_u32(&sm.s_free[i]), kSoftmaxWarps);
    }
    tc::mbar_init(smem_u32(&sm.q_ready), kSoftmaxWarps);
    tc::fence_mbar_init();
  }
  if (warp == kQkWarp) {
    tc::tmem_alloc(smem_u32(&sm.tmem_slot), kTmemCols);
    tc::tmem_relinquish();
  }
  pdl_wait();
  pdl_launch_dependents();
  tc::fence_before_sync();
  const bool dead = tc::block_gives_up(a.status);
  tc::fence_after_sync();
  const uint32_t tmem_base = sm.tmem_slot;

  // sequences without tokens belong to no tile
  for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
    if (paged::seq_length(a, b, tid == 0) > 0) continue;
    uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + b * a.ld_out);
    for (int i = tid; i < a.H * kDV / 2; i += kThreads) out[i] = 0u;
    for (int i = tid; i < a.H && a.lse != nullptr; i += kThreads) a.lse[static_cast<int64_t>(b) * a.H + i] = -INFINITY;
  }

  Cursor cur = paged::first_entry(a, blockIdx.x, kShift, 1, lane);
  if (dead) cur.left = 0;
  const int entries = static_cast<int>(cur.left);

  if (warp == kCopyWarp) {
    // ================= copies =================
    const int64_t n_rows = static_cast<int64_t>(max(a.n_pages, 1)) << a.page_shift;   // as the tensor map has them
    auto row_of = [&]() -> int {   // cache row of the tile at the cursor; past the pool (rows of zeros) if its page is not one
      if (cur.left <= 0) return 0;
      const int s0 = cur.st.first_key(cur.tile, kShift);
      const int p = a.page_table[cur.b * a.pt_stride + (s0 >> a.page_shift)];
      if (p < 0 || p >= a.n_pages) {
        if (lane == 0) paged::report_index(a.notice);
        return static_cast<int>(n_rows);
      }
      return (p << a.page_shift) + (s0 & ((1 << a.page_shift) - 1));
    };
    int row = row_of();
    int g = 0;
    for (; g < entries; ++g) {
      const int slot = g % kRing;
      const uint32_t use = static_cast<uint32_t>(g / kRing) & 1u;
      const int this_row = row;
      paged::advance(a, cur, kShift, 1);
      row = row_of();   // (its page number is on its way while this tile waits for its slot)
      if (!__all_sync(0xffffffffu, tc::mbar_wait(smem_u32(&sm.k_empty[slot]), use ^ 1u, a.status))) break;
      if (tc::elect_one()) {
        const uint32_t full = smem_u32(&sm.k_full[slot]);
        tc::mbar_expect_tx(full, kSlotBytes);
        tc::tma_load_3d(smem_u32(sm.k[slot]), &k_map, 0, this_row, 0, full);
      }
      __syncwarp();
    }
    // every copy has landed before the block ends, also if somebody gave up on a wait
    for (int i = g > kRing ? g - kRing : 0; i < g; ++i)
      (void)tc::mbar_wait(smem_u32(&sm.k_full[i % kRing]), static_cast<uint32_t>(i / kRing) & 1u, nullptr);
  } else if (warp == kQkWarp) {
    // ================= S = Q K^T =================
    if (tc::elect_one()) {
      const uint64_t dk0 = tc::smem_desc_sw128(smem_u32(sm.k), 16, 1024);
      const uint64_t dqr = tc::smem_desc_sw128(smem_u32(sm.q_rope), 16, 1024);
      constexpr uint32_t idesc = idesc_16<kF16>(kHeads, kTileKeys, 0, 0);
      constexpr uint32_t kLane16 = 16u << 16;
      bool fresh = true;
      uint32_t piece = 0;
      for (int g = 0; g < entries; ++g) {
        if (fresh && !tc::mbar_wait(smem_u32(&sm.q_ready), piece++ & 1u, a.status)) break;
        const int slot = g % kRing, buf = g & 1;
        if (!tc::mbar_wait(smem_u32(&sm.k_full[slot]), static_cast<uint32_t>(g / kRing) & 1u, a.status)) break;
        if (!tc::mbar_wait(smem_u32(&sm.s_free[buf]), (static_cast<uint32_t>(g >> 1) & 1u) ^ 1u, a.status)) break;
        tc::fence_after_sync();
        const uint64_t dk = tc::desc_advance(dk0, slot * kSlotBytes);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint32_t q_src = tmem_base + x * kLane16 + kColQ, s_dst = tmem_base + x * kLane16 + kColS + buf * kSBuf;
#pragma unroll
          for (int s = 0; s < 16; ++s)   // dims 256 x + 16 s .. + 15
            tc::umma_ts(s_dst, q_src + 8 * s, tc::desc_advance(dk, (4 * x + (s >> 2)) * kAtomBytes + (s & 3) * 32), idesc, s != 0);
#pragma unroll
          for (int s = 0; s < 2; ++s)    // dims 512 + 32 x + 16 s .. + 15
            tc::umma_ss(s_dst, tc::desc_advance(dqr, (2 * x + s) * 32), tc::desc_advance(dk, 8 * kAtomBytes + (2 * x + s) * 32), idesc, 1);
        }
        tc::umma_commit(smem_u32(&sm.s_full[buf]));
        fresh = paged::advance(a, cur, kShift, 1);
      }
    }
  } else if (warp == kPvWarp) {
    // ================= O += P V =================
    if (tc::elect_one()) {
      constexpr uint32_t idesc = idesc_16<kF16>(kHeads, 256, 0, 1);
      const uint64_t dv0 = tc::smem_desc_sw128(smem_u32(sm.k), kAtomBytes, 1024);   // MN-major view of a tile
      const uint64_t dp0 = tc::smem_desc_sw128(smem_u32(sm.k[0][8]), 16, 1024);     // P in its last column block
      bool fresh = true;
      for (int g = 0; g < entries; ++g) {
        const int slot = g % kRing;
        // (given after O of the sequence before has been read out)
        if (!tc::mbar_wait(smem_u32(&sm.p_ready[slot]), static_cast<uint32_t>(g / kRing) & 1u, a.status)) break;
        tc::fence_after_sync();
        const uint64_t dv = tc::desc_advance(dv0, slot * kSlotBytes), dp = tc::desc_advance(dp0, slot * kSlotBytes);
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int kk = 0; kk < kTileKeys / 16; ++kk)
            tc::umma_ws_ss(tmem_base + 128 * y, tc::desc_advance(dp, kk * 32), tc::desc_advance(dv, 4 * y * kAtomBytes + kk * 2048), idesc,
                           !fresh || kk > 0);
        tc::umma_commit(smem_u32(&sm.pv_done[slot]));
        tc::umma_commit(smem_u32(&sm.k_empty[slot]));
        fresh = paged::advance(a, cur, kShift, 1);
      }
    }
  } else {
    // ================= softmax, Q and O =================
    const uint32_t lane_addr = static_cast<uint32_t>(32 * warp) << 16;
    const int row_s = 16 * warp + (lane >> 2);                            // the thread's rows of S: this one and 8 more
    const int head_o = 32 * (warp & 1) + lane, half_o = warp >> 1;        // its row of O, and which half of each 256 dims
    auto fetch_q = [&](int b) {   // whole warp: 16 heads, the lanes' halves half of the first 512 dims each
      const int row = 16 * warp + (lane & 15), hi = lane >> 4;
      const bool on = row < a.H;
      const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + b * a.ld_q + static_cast<int64_t>(on ? row : 0) * kDQK);
      const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        uint4 u[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) u[j] = on ? __ldcg(src + 32 * hi + 16 * part + j) : zero;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t w[32];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            w[4 * j] = u[8 * h + j].x; w[4 * j + 1] = u[8 * h + j].y; w[4 * j + 2] = u[8 * h + j].z; w[4 * j + 3] = u[8 * h + j].w;
          }
          tc::tmem_st32(tmem_base + lane_addr + kColQ + (2 * part + h) * 32, w);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = 4 * hi + j;
        *reinterpret_cast<uint4*>(sm.q_rope + row * 128 + ((c ^ (row & 7)) << 4)) = on ? __ldcg(src + 64 + c) : zero;
      }
      tc::fence_proxy_async();
      tc::tmem_st_wait();
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(smem_u32(&sm.q_ready));
    };
    float m_used[2] = {0.f, 0.f}, l_run[2] = {0.f, 0.f};
    bool ok = true, fresh = true, from_start = cur.tile == 0, first = true;
    if (entries > 0) fetch_q(cur.b);
    for (int g = 0; g < entries; ++g) {
      const int slot = g % kRing, buf = g & 1;
      ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(smem_u32(&sm.s_full[buf]), static_cast<uint32_t>(g >> 1) & 1u, a.status));
      tc::fence_after_sync();
      float2 v[16];   // [group of eight keys j][row r] at 2 j + r: keys 8 j + 2 (lane % 4) + {0, 1}
      {
        uint32_t x[32], y[32];
        const uint32_t s_addr = tmem_base + lane_addr + kColS + buf * kSBuf;
        tc::tmem_ld_16x256b(s_addr, x);
        tc::tmem_ld_16x256b(s_addr + (16u << 16), y);
        tc::tmem_ld_wait();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(smem_u32(&sm.s_free[buf]));
#pragma unroll
        for (int j = 0; j < 16; ++j)
          v[j] = add2(make_float2(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1])),
                      make_float2(__uint_as_float(y[2 * j]), __uint_as_float(y[2 * j + 1])));
      }
      const int s0 = cur.st.first_key(cur.tile, kShift);
      const bool partial = !cur.st.all_seen(s0, kTileKeys);
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          v[2 * j + r].x *= a.scale2;
          v[2 * j + r].y *= a.scale2;
          if (partial) {
            const int s = s0 + 8 * j + 2 * (lane & 3);
            if (!cur.st.seen(s)) v[2 * j + r].x = -INFINITY;
            if (!cur.st.seen(s + 1)) v[2 * j + r].y = -INFINITY;
          }
          mx[r] = fmaxf(mx[r], fmaxf(v[2 * j + r].x, v[2 * j + r].y));
        }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 1));
        mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 2));
      }
      float alpha[2] = {1.f, 1.f};
      bool need = false;
      if (fresh) {
        m_used[0] = mx[0];
        m_used[1] = mx[1];
        l_run[0] = l_run[1] = 0.f;
      } else {
#pragma unroll
        for (int r = 0; r < 2; ++r)
          if (mx[r] > m_used[r] + kRescaleGap) {
            alpha[r] = exp2_fast(m_used[r] - mx[r]);
            m_used[r] = mx[r];
            l_run[r] *= alpha[r];
            need = true;
          }
      }
      uint32_t pk[8][2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float ref = m_used[r] > -INFINITY ? m_used[r] : 0.f;   // (a row whose scores are all -inf weighs nothing)
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 e = make_float2(exp2_fast(v[2 * j + r].x - ref), exp2_fast(v[2 * j + r].y - ref));
          sum = add2(sum, e);
          pk[j][r] = pack2<kF16>(e.x, e.y);   // 16 bits of a weight of at most 2^8; the sum is of the unrounded ones
        }
        l_run[r] += sum.x + sum.y;
      }
      {
        const int row = 16 * warp + ((lane >> 3) & 1) * 8 + (lane & 7);
        const uint32_t dst = smem_u32(sm.k[slot][8]) + row * 128;
#pragma unroll
        for (int j = 0; j < 8; j += 2)
          stmatrix_x4(dst + (((j + (lane >> 4)) ^ (row & 7)) << 4), pk[j][0], pk[j][1], pk[j + 1][0], pk[j + 1][1]);
      }
      if (partial) {   // rows that nobody sees may hold anything
        for (int r = tid >> 6; r < kTileKeys; r += 2)
          if (!cur.st.seen(s0 + r)) *reinterpret_cast<uint4*>(sm.k[slot][(tid & 63) >> 3] + r * 128 + (tid & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
      }
      tc::fence_proxy_async();
      const bool any = softmax_any(need || !ok);
      if (any) {
        // rare: O of every head times its factor, once P V of the tile before is complete
#pragma unroll
        for (int r = 0; r < 2; ++r)
          if ((lane & 3) == 0) sm.factor[row_s + 8 * r] = alpha[r];
        if (g > 0)
          ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(smem_u32(&sm.pv_done[(g - 1) % kRing]), static_cast<uint32_t>((g - 1) / kRing) & 1u, a.status));
        if (softmax_any(!ok)) break;   // all of them leave together: the named barrier has no time limit
        tc::fence_after_sync();
        const float al = sm.factor[head_o];
#pragma unroll 1
        for (int c = 0; c < 256; c += 32) {
          uint32_t o[32];
          tc::tmem_ld32(tmem_base + lane_addr + c, o);
          tc::tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * al);
          tc::tmem_st32(tmem_base + lane_addr + c, o);
        }
        tc::tmem_st_wait();
        tc::fence_before_sync();
        softmax_sync();
      }
      if (tid == 0) tc::mbar_arrive(smem_u32(&sm.p_ready[slot]));

      const bool ends = cur.tile + 1 == cur.st.count;
      const bool whole = from_start && ends;
      const int b = cur.b;
      fresh = paged::advance(a, cur, kShift, 1);
      if (!fresh && cur.left > 0) continue;

      // ---- the sequence, or this unit's part of it, is done
      if (cur.left > 0) fetch_q(cur.b);   // every Q K^T of the old one is complete
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        l_run[r] += __shfl_xor_sync(0xffffffffu, l_run[r], 1);
        l_run[r] += __shfl_xor_sync(0xffffffffu, l_run[r], 2);
        const int row = row_s + 8 * r;
        if ((lane & 3) == 0) {
          const bool some = l_run[r] > 0.f || l_run[r] != l_run[r];
          const float lse2 = some ? m_used[r] + log2f(l_run[r]) : -INFINITY;
          sm.factor[row] = some ? 1.f / l_run[r] : 0.f;
          if (row < a.H) {
            if (!whole) a.part_lse[(2 * static_cast<int64_t>(blockIdx.x) + (first ? 0 : 1)) * a.H + row] = lse2;
            else if (a.lse != nullptr) a.lse[static_cast<int64_t>(b) * a.H + row] = lse2 / paged::kLog2e;
          }
        }
      }
      ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(smem_u32(&sm.pv_done[slot]), static_cast<uint32_t>(g / kRing) & 1u, a.status));
      if (softmax_any(!ok)) break;
      tc::fence_after_sync();
      const float inv = sm.factor[head_o];
      uint16_t* out = static_cast<uint16_t*>(a.out) + b * a.ld_out + static_cast<int64_t>(head_o) * kDV + 128 * half_o;
      float* part = a.part_out + ((2 * static_cast<int64_t>(blockIdx.x) + (first ? 0 : 1)) * a.H + head_o) * kDV + 128 * half_o;
#pragma unroll 1
      for (int c = 0; c < 256; c += 32) {
        uint32_t o[32];
        tc::tmem_ld32(tmem_base + lane_addr + c, o);
        tc::tmem_ld_wait();
        if (head_o < a.H) {
          const int d = (c >> 7) * 256 + (c & 127);
          if (whole) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              uint32_t w[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) w[i] = pack2<kF16>(__uint_as_float(o[8 * j + 2 * i]) * inv, __uint_as_float(o[8 * j + 2 * i + 1]) * inv);
              *reinterpret_cast<uint4*>(out + d + 8 * j) = make_uint4(w[0], w[1], w[2], w[3]);
            }
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              *reinterpret_cast<float4*>(part + d + 4 * j) =
                  make_float4(__uint_as_float(o[4 * j]) * inv, __uint_as_float(o[4 * j + 1]) * inv, __uint_as_float(o[4 * j + 2]) * inv,
                              __uint_as_float(o[4 * j + 3]) * inv);
          }
        }
      }
      tc::fence_before_sync();   // O has been read: the next sequence's P V may begin once its first P is there
      softmax_sync();            // (and the factors have been read)
      from_start = true;
      first = false;
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == kQkWarp) tc::tmem_dealloc(tmem_base, kTmemCols);
}

}  // namespace

cudaError_t launch_paged_attn_tc(const PagedAttnArgs& a, cudaStream_t st, int64_t* n_launch) {
  static_assert(sizeof(LatentSmem) + 1024 <= 227 * 1024, "shared memory of a block");
  constexpr size_t smem = sizeof(LatentSmem) + 1024;
  CUtensorMap k_map;
  // (a pool without pages has no rows to describe; nothing is copied from it)
  const uint64_t rows = static_cast<uint64_t>(a.n_pages > 0 ? a.n_pages : 1) << a.page_shift;
  if (!make_map_bf16_tile(&k_map, a.k_pool, static_cast<uint64_t>(a.ld_k), rows, kTileKeys, kAtoms)) return cudaErrorInvalidValue;
  auto kernel = a.fp16 ? paged_latent_kernel<true> : paged_latent_kernel<false>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3(a.units), dim3(kThreads), smem, st, k_map, a);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ++*n_launch;
  return launch_paged_join(a, kShift, 1, st, n_launch);
}

}  // namespace lsa
