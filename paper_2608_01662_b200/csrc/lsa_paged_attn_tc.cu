// lsa_paged_attn over latent rows (absorbed MLA: up to 64 query heads, d_qk = 576, the value is the first 512 dims of the key
// row) on the 5th-generation tensor cores.
//
// A token's 1152 bytes meet 64 heads: 121 flop per byte, so HBM is the bound only as long as the products run on tcgen05 and
// the softmax stays beside them.  The 64 heads are the M = 64 rows of every MMA (rows of absent heads are zero).  A unit of the
// grid works through its share of the list of 64-token tiles (lsa_paged.cuh), one sequence after another:
//
//   warp 8      copies: a tile lies inside one cache page, so each half of it is one TMA box (nine column blocks of 32 rows x 128
//               bytes, 128B-swizzled), into a ring of three tiles, two slots of 36.9 KB each.  A sequence's Q (32 heads a slot)
//               goes through the ring too, ahead of its first tile.
//   warps 9, 10 S = Q K^T, a half of each tile's keys per warp, M64 N32 K16.  Q is in tensor memory (its last 64 dims in shared
//               memory), and S has two accumulation chains in the two halves of the lanes (an M = 64 accumulator uses 16 lanes of
//               each 32); two S buffers.
//   warps 0-7   softmax, four warps for each half of a tile's keys: the two partial sums are added, P = 2^(score - reference) with
//               the reference as it is, fp32 row sums, P in 16 bits into the slot's last column block, which only Q K^T reads; one
//               vote says whether the reference was good enough for every row (O is rescaled, and P worked out again, only when a
//               row's maximum has grown by more than 2^8).  At a sequence's end they move the next Q and write O.  Rows of a tile
//               that nobody sees are zeroed there before they become values: 0 x NaN is NaN.
//   warp 11     O += P V, tcgen05.mma.ws M64 N256 K16; V is the tile read MN-major, so a row is fetched once.
//
// Measured: one sequence of 524 thousand tokens 120 us (5.0 TB/s, 0.77 of a copy's rate), 64 sequences with 3.5 million 690-820 us (the
// GPU is then at its power limit, 990 W, at 1.0 to 1.4 of its 1.97 GHz: a tile takes 2160 or 2500 cycles and the same time), one of a
// few hundred tokens 11 us, of which 4 pass before the first tile is there and 3 to 4 in the kernel that joins.  Tiles of 32 tokens took
// 1475 cycles each: the softmax's chain from one to the next, not its work.  One issuing thread for both halves of Q K^T stalls for
// some 400 cycles behind each commit (the first sequence 122.5 us instead of 118.5, the 64 733 instead of 690).
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
constexpr int kHalfKeys = kTileKeys / 2, kGroups = kHalfKeys / 8;   // keys of a ring slot, of a softmax warp; in fragments of eight
constexpr int kAtomBytes = kHalfKeys * 128;
constexpr int kSlotBytes = kAtoms * kAtomBytes;
constexpr int kRing = 3;                                            // tiles, two slots each
constexpr int kSoftmaxWarps = 8, kCopyWarp = 8, kQkWarp = 9, kPvWarp = 11, kThreads = 384;
constexpr int kSoftmaxThreads = 32 * kSoftmaxWarps;
constexpr uint32_t kTmemCols = 512, kColQ = 256, kColS = 384, kSBuf = 64;

struct LatentSmem {
  alignas(1024) uint8_t k[2 * kRing][kAtoms][kAtomBytes];
  alignas(1024) uint8_t q_rope[kHeads * 128];
  alignas(8) uint64_t k_full[2 * kRing], k_empty[2 * kRing], p_ready[kRing], pv_done[kRing], s_full[4], s_free[4], q_ready;
  uint32_t tmem_slot;
  float factor[kHeads];        // of a rescaling of O; at a sequence's end 1 / l
  float half_max[2][kHeads];   // [half of a tile's keys][row]: its maximum, where both halves have to know it
  float half_sum[kHeads];      // row sums of the second halves
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

// K-major operand of 64-byte rows (32 elements), 64-byte swizzle: the 16-byte units of row r are XORed with (r / 2) % 4; groups of eight
// rows `sbo` bytes apart.
__device__ __forceinline__ uint64_t smem_desc_sw64(uint32_t addr, uint32_t sbo) {
  return (tc::smem_desc_sw128(addr, 16, sbo) & ~(7ull << 61)) | (4ull << 61);
}

template <bool kF16>
__global__ void __launch_bounds__(kThreads, 1) paged_latent_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap q_map,
                                                                   PagedAttnArgs p) {
  extern __shared__ uint8_t smem_raw[];
  LatentSmem& sm = *reinterpret_cast<LatentSmem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  constexpr float kLift = paged::kLift<kF16>, kGap = paged::kRescaleGap + kLift;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);

  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
    for (int i = 0; i < 2 * kRing; ++i) {
      tc::mbar_init(smem_u32(&sm.k_full[i]), 1);
      tc::mbar_init(smem_u32(&sm.k_empty[i]), 1);
    }
    for (int i = 0; i < kRing; ++i) {
      tc::mbar_init(smem_u32(&sm.p_ready[i]), 1);
      tc::mbar_init(smem_u32(&sm.pv_done[i]), 1);
    }
    for (int i = 0; i < 4; ++i) {
      tc::mbar_init(smem_u32(&sm.s_full[i]), 1);
      tc::mbar_init(smem_u32(&sm.s_free[i]), kSoftmaxWarps / 2);
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
  const bool raised = tc::status_raised(p.status);
  Cursor cur = paged::first_entry(p, blockIdx.x, kShift, 1, lane);
  const bool dead = __syncthreads_or(raised) != 0;   // the same in all threads, as in tc::block_gives_up
  tc::fence_after_sync();
  const uint32_t tmem_base = sm.tmem_slot;
  const int entries = dead ? 0 : cur.left;
  if (dead) cur.left = 0;

  if (warp == kCopyWarp) {
    // ================= copies =================
    const int64_t n_rows = static_cast<int64_t>(max(p.n_pages, 1)) << p.page_shift;   // as the tensor map has them
    auto row_of = [&]() -> int {   // cache row of the tile at the cursor; past the pool (rows of zeros) if its page is not one
      if (cur.left <= 0) return 0;
      const int s0 = cur.st.first_key(cur.tile, kShift);
      const int page = p.page_table[cur.b * p.pt_stride + (s0 >> p.page_shift)];
      if (page < 0 || page >= p.n_pages) {
        if (lane == 0) paged::report_index(p.notice);
        return static_cast<int>(n_rows);
      }
      return (page << p.page_shift) + (s0 & ((1 << p.page_shift) - 1));
    };
    // Items of the ring, two slots each: Q of a sequence (heads 0-31, 32-63), then its tiles.
    int row = row_of(), pair = 0, issued = 0;
    uint32_t use = 0;
    bool alive = true, fresh = true;
    for (int g = 0; g < entries && alive; ++g) {
      const int this_row = row, b = cur.b;
      const bool q_first = fresh;
      fresh = paged::advance(p, cur, kShift, 1);
      row = row_of();   // (its page number is on its way while this tile waits for its slots)
      for (int item = q_first ? 0 : 1; item < 2 && alive; ++item) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          alive = alive && __all_sync(0xffffffffu, tc::mbar_wait(smem_u32(&sm.k_empty[2 * pair + h]), use ^ 1u, p.status));
          if (!alive) break;
          if (tc::elect_one()) {
            const uint32_t full = smem_u32(&sm.k_full[2 * pair + h]), dst = smem_u32(sm.k[2 * pair + h]);
            tc::mbar_expect_tx(full, kSlotBytes);
            if (item == 0) tc::tma_load_4d(dst, &q_map, 0, 32 * h, 0, b, full);
            else tc::tma_load_3d(dst, &k_map, 0, this_row + kHalfKeys * h, 0, full);
          }
          __syncwarp();
          ++issued;
        }
        if (++pair == kRing) {
          pair = 0;
          use ^= 1u;
        }
      }
    }
    // every copy has landed before the block ends, also if somebody gave up on a wait
    for (int i = max(issued - 2 * kRing, 0); i < issued; ++i)
      (void)tc::mbar_wait(smem_u32(&sm.k_full[i % (2 * kRing)]), static_cast<uint32_t>(i / (2 * kRing)) & 1u, nullptr);
  } else if (warp == kQkWarp || warp == kQkWarp + 1) {
    // ================= S = Q K^T =================
    if (tc::elect_one()) {
      const uint64_t dk0 = tc::smem_desc_sw128(smem_u32(sm.k), 16, 1024);
      const uint64_t dqr = tc::smem_desc_sw128(smem_u32(sm.q_rope), 16, 1024);
      constexpr uint32_t idesc = idesc_16<kF16>(kHeads, kHalfKeys, 0, 0);
      constexpr uint32_t kLane16 = 16u << 16;
      const int h = warp - kQkWarp;   // the half of the tiles
      bool fresh = true, ok = true;
      uint32_t piece = 0, use = 0;
      int pair = 0;
      auto next = [&]() {
        if (++pair == kRing) {
          pair = 0;
          use ^= 1u;
        }
      };
      for (int g = 0; g < entries && ok; ++g) {
        if (fresh) {
          if (!tc::mbar_wait(smem_u32(&sm.q_ready), piece++ & 1u, p.status)) break;
          tc::mbar_arrive(smem_u32(&sm.k_empty[2 * pair + h]));   // Q has left its slots
          next();
        }
        const int buf = g & 1;
        ok = tc::mbar_wait(smem_u32(&sm.k_full[2 * pair + h]), use, p.status) &&
             tc::mbar_wait(smem_u32(&sm.s_free[2 * buf + h]), (static_cast<uint32_t>(g >> 1) & 1u) ^ 1u, p.status);
        if (!ok) break;
        tc::fence_after_sync();
        const uint64_t dk = tc::desc_advance(dk0, (2 * pair + h) * kSlotBytes);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint32_t q_src = tmem_base + x * kLane16 + kColQ, s_dst = tmem_base + x * kLane16 + kColS + buf * kSBuf + kHalfKeys * h;
#pragma unroll
          for (int s = 0; s < 16; ++s)   // dims 256 x + 16 s .. + 15
            tc::umma_ts(s_dst, q_src + 8 * s, tc::desc_advance(dk, (4 * x + (s >> 2)) * kAtomBytes + (s & 3) * 32), idesc, s != 0);
#pragma unroll
          for (int s = 0; s < 2; ++s)    // dims 512 + 32 x + 16 s .. + 15
            tc::umma_ss(s_dst, tc::desc_advance(dqr, (2 * x + s) * 32), tc::desc_advance(dk, 8 * kAtomBytes + (2 * x + s) * 32), idesc, 1);
        }
        tc::umma_commit(smem_u32(&sm.s_full[2 * buf + h]));
        next();
        fresh = paged::advance(p, cur, kShift, 1);
      }
    }
  } else if (warp == kPvWarp) {
    // ================= O += P V =================
    if (entries == 0 && lane == 0) p.parts[blockIdx.x] = make_int4(0, 0, 0, 0);
    // sequences without tokens belong to no tile: their results, while the first tile is on its way
    for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
      if (paged::seq_length(p, b, lane == 0) > 0) continue;
      uint4* out = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + b * p.ld_out);
      for (int i = lane; i < p.H * kDV / 8; i += 32) out[i] = make_uint4(0u, 0u, 0u, 0u);
      for (int i = lane; i < p.H && p.lse != nullptr; i += 32) p.lse[static_cast<int64_t>(b) * p.H + i] = -INFINITY;
    }
    __syncwarp();
    if (tc::elect_one()) {
      constexpr uint32_t idesc = idesc_16<kF16>(kHeads, 256, 0, 1);
      const uint64_t dv0 = tc::smem_desc_sw128(smem_u32(sm.k), kAtomBytes, 1024);   // MN-major view of a slot
      const uint64_t dp0 = smem_desc_sw64(smem_u32(sm.k[0][8]), 512);               // P in its last column block
      bool fresh = true;
      int pair = 0, turn = 0;   // ring position of the tile; its number, modulo kRing
      uint32_t use = 0;
      for (int g = 0; g < entries; ++g) {
        if (fresh && ++pair == kRing) pair = 0;   // (Q)
        // (given after O of the sequence before has been read out)
        if (!tc::mbar_wait(smem_u32(&sm.p_ready[turn]), use, p.status)) break;
        tc::fence_after_sync();
        // the softmax warps give a sequence's last slots free: they may stage O there
        const bool last = cur.tile + 1 == cur.st.count || cur.left == 1;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint64_t dv = tc::desc_advance(dv0, (2 * pair + h) * kSlotBytes), dp = tc::desc_advance(dp0, (2 * pair + h) * kSlotBytes);
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int kk = 0; kk < kHalfKeys / 16; ++kk)
              tc::umma_ws_ss(tmem_base + 128 * y, tc::desc_advance(dp, kk * 32), tc::desc_advance(dv, 4 * y * kAtomBytes + kk * 2048), idesc,
                             !fresh || h > 0 || kk > 0);
          if (h == 1) tc::umma_commit(smem_u32(&sm.pv_done[turn]));
          if (!last) tc::umma_commit(smem_u32(&sm.k_empty[2 * pair + h]));
        }
        if (++pair == kRing) pair = 0;
        if (++turn == kRing) {
          turn = 0;
          use ^= 1u;
        }
        fresh = paged::advance(p, cur, kShift, 1);
      }
    }
  } else {
    // ================= softmax, Q and O =================
    const int quarter = warp & 3, half = warp >> 2;
    const uint32_t lane_addr = static_cast<uint32_t>(32 * quarter) << 16;
    const int row_s = 16 * quarter + (lane >> 2);                           // the thread's rows of S: this one and 8 more
    const int head_o = 32 * (quarter & 1) + lane, half_o = quarter >> 1;    // its row of O, and which half of each 256 dims
    const int col_o = 128 * half;                                           // its columns of O: dims 256 half + 128 half_o + 0 .. 127
    int pair = 0, turn = 0;            // ring position of the item; number of the tile, modulo kRing
    uint32_t use = 0, turn_use = 0;    // parities of their uses
    auto next_item = [&]() {
      if (++pair == kRing) {
        pair = 0;
        use ^= 1u;
      }
    };
    // Q from its slots to tensor memory, two dims a column: of 16 heads, the lanes' halves have 256 dims each, the warps' halves 128 of them
    auto move_q = [&]() -> bool {
      const int row = 16 * quarter + (lane & 15), hi = lane >> 4, r = row & 31;
      const int at = 2 * pair + (quarter >> 1);
      if (!__all_sync(0xffffffffu, tc::mbar_wait(smem_u32(&sm.k_full[at]), use, p.status))) return false;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t w[32];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const uint4 u = *reinterpret_cast<const uint4*>(sm.k[at][4 * hi + 2 * half + h] + r * 128 + ((c ^ (r & 7)) << 4));
          w[4 * c] = u.x; w[4 * c + 1] = u.y; w[4 * c + 2] = u.z; w[4 * c + 3] = u.w;
        }
        tc::tmem_st32(tmem_base + lane_addr + kColQ + (2 * half + h) * 32, w);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int c = ((4 * half + 2 * hi + j) ^ (r & 7)) << 4;
        *reinterpret_cast<uint4*>(sm.q_rope + row * 128 + c) = *reinterpret_cast<const uint4*>(sm.k[at][8] + r * 128 + c);
      }
      tc::fence_proxy_async();   // q_rope is read, and the slots are written, by the async proxy
      tc::tmem_st_wait();
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(smem_u32(&sm.q_ready));
      next_item();
      return true;
    };
    float m_used[2] = {0.f, 0.f}, l_run[2] = {0.f, 0.f};   // references of rows row_s and row_s + 8, in log2 units; the thread's share of their sums
    bool ok = true, fresh = true, from_start = cur.tile == 0, first = true;
    if (entries > 0) ok = move_q();
    for (int g = 0; g < entries; ++g) {
      const int buf = g & 1;
      const int s0 = cur.st.first_key(cur.tile, kShift) + kHalfKeys * half;
      const bool partial = !cur.st.all_seen(s0, kHalfKeys);
      ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(smem_u32(&sm.s_full[2 * buf + half]), static_cast<uint32_t>(g >> 1) & 1u, p.status));
      tc::fence_after_sync();
      float2 v[2 * kGroups];   // [group of eight keys j][row r] at 2 j + r: keys 8 j + 2 (lane % 4) + {0, 1} of the half
      {
        uint32_t x[4 * kGroups], y[4 * kGroups];
        const uint32_t s_addr = tmem_base + lane_addr + kColS + buf * kSBuf + kHalfKeys * half;
        tc::tmem_ld_16x256b(s_addr, x);
        tc::tmem_ld_16x256b(s_addr + (16u << 16), y);
        tc::tmem_ld_wait();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(smem_u32(&sm.s_free[2 * buf + half]));
#pragma unroll
        for (int j = 0; j < 2 * kGroups; ++j)
          v[j] = add2(make_float2(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1])),
                      make_float2(__uint_as_float(y[2 * j]), __uint_as_float(y[2 * j + 1])));
      }
      if (partial) {
#pragma unroll
        for (int j = 0; j < kGroups; ++j)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int s = s0 + 8 * j + 2 * (lane & 3);
            if (!cur.st.seen(s)) v[2 * j + r].x = -INFINITY;
            if (!cur.st.seen(s + 1)) v[2 * j + r].y = -INFINITY;
          }
        // rows that nobody sees may hold anything
        for (int r = (tid >> 6) & 1; r < kHalfKeys; r += 2)
          if (!cur.st.seen(s0 + r))
            *reinterpret_cast<uint4*>(sm.k[2 * pair + half][(tid & 63) >> 3] + r * 128 + (tid & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
      }
      float mx[2];   // of the thread's values, then of the rows'
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float x = fmaxf(v[r].x, v[r].y);
#pragma unroll
        for (int j = 1; j < kGroups; ++j) x = fmaxf(x, fmaxf(v[2 * j + r].x, v[2 * j + r].y));
        mx[r] = x * p.scale2;
      }
      auto row_max = [&]() {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 1));
          mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 2));
          if ((lane & 3) == 0) sm.half_max[half][row_s + 8 * r] = mx[r];
        }
        softmax_sync();
#pragma unroll
        for (int r = 0; r < 2; ++r) mx[r] = fmaxf(mx[r], sm.half_max[half ^ 1][row_s + 8 * r]);
      };
      bool need = false;
      if (fresh) {
        row_max();
        m_used[0] = mx[0] - kLift;
        m_used[1] = mx[1] - kLift;
        l_run[0] = l_run[1] = 0.f;
      } else {
        need = mx[0] > m_used[0] + kGap || mx[1] > m_used[1] + kGap;
      }
      float sum[2];
      auto work_out_p = [&]() {
        uint32_t pk[kGroups][2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float ref = m_used[r] > -INFINITY ? m_used[r] : 0.f;   // (a row whose scores are all -inf weighs nothing)
          const float2 scale = make_float2(p.scale2, p.scale2), minus = make_float2(-ref, -ref);
          float2 sum2 = make_float2(0.f, 0.f);
#pragma unroll
          for (int j = 0; j < kGroups; ++j) {
            float2 e = fma2(v[2 * j + r], scale, minus);
            e.x = exp2_fast(e.x);
            e.y = exp2_fast(e.y);
            sum2 = add2(sum2, e);
            pk[j][r] = pack2<kF16>(e.x, e.y);   // the sum is of the unrounded ones
          }
          sum[r] = sum2.x + sum2.y;
        }
        const int row = 16 * quarter + ((lane >> 3) & 1) * 8 + (lane & 7);
        const uint32_t dst = smem_u32(sm.k[2 * pair + half][8]) + row * 64;
#pragma unroll
        for (int j = 0; j < kGroups; j += 2)
          stmatrix_x4(dst + (((j + (lane >> 4)) ^ ((row >> 1) & 3)) << 4), pk[j][0], pk[j][1], pk[j + 1][0], pk[j + 1][1]);
      };
      work_out_p();
      tc::fence_proxy_async();
      if (softmax_any(need || !ok)) {
        if (softmax_any(!ok)) break;   // all of them leave together: the named barrier has no time limit
        // rare: O of every head times its factor, once P V of the tile before is complete, and P once more
        row_max();
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float alpha = 1.f;
          if (mx[r] > m_used[r] + kGap) {
            alpha = exp2_fast(m_used[r] - (mx[r] - kLift));
            m_used[r] = mx[r] - kLift;
          }
          l_run[r] *= alpha;
          if (half == 0 && (lane & 3) == 0) sm.factor[row_s + 8 * r] = alpha;
        }
        const int before = turn == 0 ? kRing - 1 : turn - 1;   // (there is a tile before: a first one needs nothing)
        ok = __all_sync(0xffffffffu, tc::mbar_wait(smem_u32(&sm.pv_done[before]), turn == 0 ? turn_use ^ 1u : turn_use, p.status));
        if (softmax_any(!ok)) break;
        tc::fence_after_sync();
        const float al = sm.factor[head_o];
#pragma unroll 1
        for (int c = col_o; c < col_o + 128; c += 32) {
          uint32_t o[32];
          tc::tmem_ld32(tmem_base + lane_addr + c, o);
          tc::tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * al);
          tc::tmem_st32(tmem_base + lane_addr + c, o);
        }
        tc::tmem_st_wait();
        work_out_p();
        tc::fence_proxy_async();
        tc::fence_before_sync();
        softmax_sync();
      }
      if (tid == 0) tc::mbar_arrive(smem_u32(&sm.p_ready[turn]));
      l_run[0] += sum[0];
      l_run[1] += sum[1];

      const int this_turn = turn, this_pair = pair;
      const uint32_t this_use = turn_use;
      if (++turn == kRing) {
        turn = 0;
        turn_use ^= 1u;
      }
      next_item();
      const bool ends = cur.tile + 1 == cur.st.count;
      if (!ends && cur.left > 1) {
        ++cur.tile;
        --cur.left;
        fresh = false;
        continue;
      }

      // ---- the sequence, or this unit's part of it, is done
      const bool whole = from_start && ends;
      const int b = cur.b;
      if (cur.left == 1 && tid == 0) paged::say_parts(p, blockIdx.x, cur, from_start, first);
      fresh = paged::advance(p, cur, kShift, 1);
      if (cur.left > 0) ok = move_q();   // every Q K^T of the old one is complete
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        l_run[r] += __shfl_xor_sync(0xffffffffu, l_run[r], 1);
        l_run[r] += __shfl_xor_sync(0xffffffffu, l_run[r], 2);
        if (half == 1 && (lane & 3) == 0) sm.half_sum[row_s + 8 * r] = l_run[r];
      }
      softmax_sync();
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int row = row_s + 8 * r;
        if (half == 0 && (lane & 3) == 0) {
          const float l = l_run[r] + sm.half_sum[row];
          const bool some = l > 0.f || l != l;
          const float lse2 = some ? m_used[r] + log2f(l) : -INFINITY;
          sm.factor[row] = some ? 1.f / l : 0.f;
          if (row < p.H) {
            if (!whole) p.part_lse[(2 * blockIdx.x + (first ? 0 : 1)) * kHeads + row] = lse2;
            else if (p.lse != nullptr) p.lse[static_cast<int64_t>(b) * p.H + row] = lse2 / paged::kLog2e;
          }
        }
      }
      ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(smem_u32(&sm.pv_done[this_turn]), this_use, p.status));
      if (softmax_any(!ok)) break;
      tc::fence_after_sync();
      const float inv = sm.factor[head_o];
      const int dim0 = 256 * half + 128 * half_o;
      uint8_t* stage = &sm.k[2 * this_pair][0][0];   // whole results: rows of 1024 bytes, 16-byte units XORed with the row, over two slots
      float* part = p.part_out + ((2 * static_cast<int64_t>(blockIdx.x) + (first ? 0 : 1)) * kDV + dim0) * kHeads + 4 * head_o;
#pragma unroll 1
      for (int c = 0; c < 128; c += 32) {
        uint32_t o[32];
        tc::tmem_ld32(tmem_base + lane_addr + col_o + c, o);
        tc::tmem_ld_wait();
        if (whole) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack2<kF16>(__uint_as_float(o[8 * j + 2 * i]) * inv, __uint_as_float(o[8 * j + 2 * i + 1]) * inv);
            *reinterpret_cast<uint4*>(stage + head_o * 1024 + ((((dim0 + c) / 8 + j) ^ (head_o & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else if (head_o < p.H) {   // a part: four dims of each head, the lanes' heads side by side (a row of its own per lane took 10 thousand cycles to store)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            *reinterpret_cast<float4*>(part + (c + 4 * j) * kHeads) =
                make_float4(__uint_as_float(o[4 * j]) * inv, __uint_as_float(o[4 * j + 1]) * inv, __uint_as_float(o[4 * j + 2]) * inv,
                            __uint_as_float(o[4 * j + 3]) * inv);
        }
      }
      tc::fence_before_sync();   // O has been read: the next sequence's P V may begin once its first P is there
      softmax_sync();            // (and the factors have been read)
      if (whole) {
        uint16_t* out = static_cast<uint16_t*>(p.out) + b * p.ld_out;
        for (int i = tid; i < p.H * (kDV / 8); i += kSoftmaxThreads) {
          const int row = i >> 6, u = i & 63;
          *reinterpret_cast<uint4*>(out + 8 * i) = *reinterpret_cast<const uint4*>(stage + row * 1024 + ((u ^ (row & 7)) << 4));
        }
        tc::fence_proxy_async();
        softmax_sync();
      }
      if (tid < 2) tc::mbar_arrive(smem_u32(&sm.k_empty[2 * this_pair + tid]));
      from_start = true;
      first = false;
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == kQkWarp) tc::tmem_dealloc(tmem_base, kTmemCols);
}

// ---- parts of a sequence that several units worked on
// Weights 2^(lse_i - max) / sum over the parts, a fixed order of addition.  A part is [dim / 4][64 heads][4 dims], so a thread has one
// head and a warp's loads are 512 bytes.  A round of a block is 64 dims where a sequence has a few parts, 16 with up to eight parts of
// many sequences, and else (one long sequence is 148 parts of 128 KB, which all SMs have to fetch together) four, four threads
// sharing a head's parts.  (16 sequences of 777 tokens, 7 parts each: 23.8 us by fours, 19.2 so; by 16 for up to 16 parts 23.2,
// the loop is then as long for all.)  Two blocks an SM: at 64 registers, four of them, the loads are no longer on their way together
// (one sequence of 8000 tokens 15.3 us, 20.6).
constexpr int kJoinThreads = paged::kJoinThreads, kWays = 4;
constexpr int kFewParts = 4, kFewDims = 64, kSomeParts = 8, kSomeDims = 16, kSomeOwners = 8, kManyDims = 4, kManyAtOnce = 10;
template <int V>
struct IntC { static constexpr int value = V; };
__device__ __forceinline__ void add(float4& x, float w, const float4& y) { x.x += w * y.x; x.y += w * y.y; x.z += w * y.z; x.w += w * y.w; }

template <bool kF16>
__global__ void __launch_bounds__(kJoinThreads, 2) paged_latent_join_kernel(PagedAttnArgs a) {
  __shared__ paged::JoinList list;
  __shared__ uint32_t tile[kHeads][kFewDims / 2 + 1];
  __shared__ float4 red[kWays][kHeads];
  __shared__ float2 stats[kWays][kHeads];   // {maximum, sum} of a thread's parts
  const int tid = threadIdx.x, head = tid & 63, way = tid >> 6;
  pdl_wait();
  pdl_launch_dependents();
  auto dims_of = [](int n, int owners) { return n <= kFewParts ? kFewDims : n <= kSomeParts && owners >= kSomeOwners ? kSomeDims : kManyDims; };
  auto rounds_of = [&](int n, int owners) { return n == 0 ? 0 : kDV / dims_of(n, owners); };
  int4 mine;
  int begins, owners;
  const int total = paged::join_list(a, list, tid, &mine, &begins, &owners, rounds_of);
  for (int it = blockIdx.x; it < total; it += gridDim.x) {   // block-uniform
    paged::join_find(list, tid, it, mine, begins, owners, rounds_of);
    const int4 own = list.own;
    const int n = own.x, round = list.round, unit = list.unit;
    auto slot = [&](int i) -> int64_t { return i == 0 ? own.w : 2 * (unit + i); };
    uint16_t* out = static_cast<uint16_t*>(a.out) + own.y * a.ld_out;
    auto finish = [&](float m, float den) -> float {   // 1 / sum; the log-sum-exp of the head by one thread
      const bool some = den > 0.f || den != den;
      if (round == 0 && way == 0 && head < a.H && a.lse != nullptr)
        a.lse[static_cast<int64_t>(own.y) * a.H + head] = some ? (m + log2f(den)) / paged::kLog2e : -INFINITY;
      return some ? 1.f / den : 0.f;
    };
    auto several = [&](auto parts_c, auto dims_c) {   // up to so many parts, so many dims
      constexpr int kParts = decltype(parts_c)::value, kDims = decltype(dims_c)::value, kMine = kDims / kWays;
      float w[kParts], m = -INFINITY, den = 0.f;
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        w[i] = i < n && head < a.H ? __ldcg(a.part_lse + slot(i) * kHeads + head) : -INFINITY;
        m = fmaxf(m, w[i]);
      }
      const float ref = m > -INFINITY ? m : 0.f;
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        w[i] = exp2f(w[i] - ref);
        den += w[i];
      }
      const float inv = finish(m, den);
      float4 x[kMine / 4] = {};
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        if (i < n && head < a.H) {
          const float* src = a.part_out + (slot(i) * kDV + round * kDims + way * kMine) * kHeads + 4 * head;
          const float wi = w[i] * inv;
#pragma unroll
          for (int j = 0; j < kMine / 4; ++j) add(x[j], wi, __ldcg(reinterpret_cast<const float4*>(src + 4 * j * kHeads)));
        }
      }
#pragma unroll
      for (int j = 0; j < kMine / 4; ++j) {
        tile[head][way * kMine / 2 + 2 * j] = pack2<kF16>(x[j].x, x[j].y);
        tile[head][way * kMine / 2 + 2 * j + 1] = pack2<kF16>(x[j].z, x[j].w);
      }
      __syncthreads();
      for (int i = tid; i < a.H * (kDims / 2); i += kJoinThreads) {
        const int row = i / (kDims / 2), d = i % (kDims / 2);
        *reinterpret_cast<uint32_t*>(out + row * kDV + round * kDims + 2 * d) = tile[row][d];
      }
    };
    const int dims = dims_of(n, owners);
    if (dims == kFewDims) {
      several(IntC<kFewParts>{}, IntC<kFewDims>{});
    } else if (dims == kSomeDims) {
      several(IntC<kSomeParts>{}, IntC<kSomeDims>{});
    } else {
      // the thread's parts, kManyAtOnce on their way at a time, relative to their maximum so far
      float m = -INFINITY, den = 0.f;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      const float* src = a.part_out + static_cast<int64_t>(round) * kManyDims * kHeads + 4 * head;
      for (int i0 = way; i0 < n; i0 += kManyAtOnce * kWays) {
        float4 y[kManyAtOnce];
        float w[kManyAtOnce], top = m;
#pragma unroll
        for (int k = 0; k < kManyAtOnce; ++k) {
          const int i = i0 + k * kWays;
          w[k] = -INFINITY;
          y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (i < n && head < a.H) {
            w[k] = __ldcg(a.part_lse + slot(i) * kHeads + head);
            y[k] = __ldcg(reinterpret_cast<const float4*>(src + slot(i) * kDV * kHeads));
          }
        }
#pragma unroll
        for (int k = 0; k < kManyAtOnce; ++k) top = fmaxf(top, w[k]);
        const float ref = top > -INFINITY ? top : 0.f, old = exp2f(m - ref);
        m = top;
        den *= old;
        x = make_float4(x.x * old, x.y * old, x.z * old, x.w * old);
#pragma unroll
        for (int k = 0; k < kManyAtOnce; ++k) {
          const float e = exp2f(w[k] - ref);
          den += e;
          add(x, e, y[k]);
        }
      }
      red[way][head] = x;
      stats[way][head] = make_float2(m, den);
      __syncthreads();
      if (way == 0) {
        float top = m;
#pragma unroll
        for (int i = 1; i < kWays; ++i) top = fmaxf(top, stats[i][head].x);
        const float ref = top > -INFINITY ? top : 0.f;
        x = make_float4(0.f, 0.f, 0.f, 0.f);
        den = 0.f;
#pragma unroll
        for (int i = 0; i < kWays; ++i) {
          const float2 s = stats[i][head];
          const float f = exp2f(s.x - ref);
          den += f * s.y;
          add(x, f, red[i][head]);
        }
        const float inv = finish(top, den);
        if (head < a.H)
          *reinterpret_cast<uint2*>(out + head * kDV + round * kManyDims) = make_uint2(pack2<kF16>(x.x * inv, x.y * inv), pack2<kF16>(x.z * inv, x.w * inv));
      }
    }
  }
}

}  // namespace

cudaError_t launch_paged_attn_tc(const PagedAttnArgs& a, cudaStream_t st, int64_t* n_launch) {
  static_assert(sizeof(LatentSmem) + 1024 <= 227 * 1024, "shared memory of a block");
  constexpr size_t smem = sizeof(LatentSmem) + 1024;
  CUtensorMap k_map, q_map;
  // (a pool without pages has no rows to describe; nothing is copied from it)
  const uint64_t rows = static_cast<uint64_t>(a.n_pages > 0 ? a.n_pages : 1) << a.page_shift;
  if (!make_map_bf16_tile(&k_map, a.k_pool, static_cast<uint64_t>(a.ld_k), rows, kHalfKeys, kAtoms) ||
      !make_map_16bit_groups(&q_map, a.q, kDQK, static_cast<uint64_t>(a.H), static_cast<uint64_t>(a.batch), static_cast<uint64_t>(a.ld_q), kHeads / 2))
    return cudaErrorInvalidValue;
  auto kernel = a.fp16 ? paged_latent_kernel<true> : paged_latent_kernel<false>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3(a.units), dim3(kThreads), smem, st, k_map, q_map, a);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ++*n_launch;
  auto join = a.fp16 ? paged_latent_join_kernel<true> : paged_latent_join_kernel<false>;
  e = launch_pdl(join, dim3(2 * a.units), dim3(kJoinThreads), 0, st, a);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e == cudaSuccess) ++*n_launch;
  return e;
}

}  // namespace lsa
