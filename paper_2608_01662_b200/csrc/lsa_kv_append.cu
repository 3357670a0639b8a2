// lsa_kv_append: new tokens of a batch of sequences into the rows of a paged cache.
//
// A block takes one token: its query heads, key heads and value heads are rows of D elements.  A thread keeps one place
// within a row for all rows that it visits: 16 dims, two 16-byte vectors.  In the rotated part these are the two halves of
// eight pairs (x cos - y sin, y cos + x sin), so the angles' cosines and sines are fetched once per thread, not once per head; a
// row's threads are consecutive lanes, so the largest element of an e4m3 row is a few shuffles.
//
// Bound: HBM for prompts (read and write once: 17 thousand tokens, 32 query and 8 KV heads of 128, 70 us, 0.94 of a copy's rate; 9871
// tokens, 64 query heads, e4m3 caches 67 us, 0.88), a launch and the chain length -> page -> row for decode steps (3 to 5 us).  Rows are
// on their way before the token's place is known, and no load stands behind a branch (with branches around the loads: 90 us, not 69).
// Between the two, and for narrow tokens, it is the chain of a block, which lives for one token: 5000 tokens of latent rows 133 us with 64
// heads (0.86 of a copy's rate), 51 with 16 (0.60); 400 tokens 15.3 (0.60) and 4.9 (0.50); 5000 of 32 over 8 heads 24.5 (0.78), into
// codes 27.9 (0.63).
#include <algorithm>

#include "lsa_paged.cuh"

namespace lsa {

namespace {

template <typename T>
struct Two;
template <>
struct Two<__nv_bfloat16> {
  __device__ static float2 get(uint32_t w) { return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&w)); }
  __device__ static uint32_t put(float x, float y) { return pack_bf16(x, y); }
};
template <>
struct Two<__half> {
  __device__ static float2 get(uint32_t w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }
  __device__ static uint32_t put(float x, float y) {
    __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<uint32_t*>(&h);
  }
};

template <typename T>
__device__ __forceinline__ void unpack8(const uint4& u, float* x) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = Two<T>::get(w[j]);
    x[2 * j] = f.x;
    x[2 * j + 1] = f.y;
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float* x) {
  return make_uint4(Two<T>::put(x[0], x[1]), Two<T>::put(x[2], x[3]), Two<T>::put(x[4], x[5]), Two<T>::put(x[6], x[7]));
}
// Eight codes of value / scale: round to nearest even, saturating.  inv is 1 / scale, correctly rounded; q = x inv, then q + (x - q scale) inv
// with the remainder in one fma is then the correctly rounded quotient (Markstein 1990), a third of the instructions of a division
// each.  The remainder is a multiple of the last places of q and scale and has to be a number of fp32, whose smallest is 2^-149: for the
// quotients that codes are told apart by, from 2^-11 on, 2^-34 times a scale's 2^-113 still is.  For scales below 2^-90 it is divided.
__device__ __forceinline__ uint2 codes8(const float* x, float scale, float inv) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t r = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float2 v = make_float2(x[4 * h + 2 * j], x[4 * h + 2 * j + 1]);
      if (inv >= 1.17549435e-38f && inv <= 0x1p90f) {
        const float p = v.x * inv, q = v.y * inv;
        v = make_float2(fmaf(fmaf(-p, scale, v.x), inv, p), fmaf(fmaf(-q, scale, v.y), inv, q));
      } else {   // a scale near either end of fp32 (its reciprocal is not a normal number, or the remainder none), infinite or NaN
        v = make_float2(__fdiv_rn(v.x, scale), __fdiv_rn(v.y, scale));
      }
      r |= static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3)) << (16 * j);
    }
    w[h] = r;
  }
  return make_uint2(w[0], w[1]);
}

// The length of sequence i after the call.
__device__ __forceinline__ int32_t new_length(const KvAppendArgs& a, int i) {
  const int32_t t0 = a.tok_start[i], t1 = a.tok_start[i + 1];
  if (t0 < 0 || t1 < t0 || t1 > a.n_tok) paged::report_index(a.notice);
  return a.ctx_len[i] + max(t1 - t0, 0);
}

// Threads of a block.  A token's rows are shared by 64 threads (288 for the latent rows of 36 places), so that many tokens are on an SM
// at a time; where there is at most one token an SM, and its rows are more than those threads have on their way, by 512 (576).  96
// query and 8 KV heads of 128: 148 tokens 3.9 us by 512 threads, 5.2 by 64; 250 tokens 6.7, 5.2; 32 query heads: 148 tokens 3.3, 2.7.
template <int D>
constexpr int kFewTokens = D == 576 ? 576 : 512;
template <int D>
constexpr int kManyTokens = D == 576 ? 288 : 64;
// Query rows that a thread has on their way at a time: four, or two where the block's threads then have all of them, and more blocks
// fit an SM (latent rows of 16 heads: 5000 tokens 65 us by four, 51 by two, 250 tokens 4.2, 4.7; 64 heads, 5000 tokens: 134, 139).  A
// block of 288 threads is nine warps, so that of two one SM partition has five: they fit with 96 registers each, which is what a bound of
// two blocks of ten warps gives.  Three blocks with two rows a thread have 64 registers: 32 to 52 bytes a thread go to memory and back,
// once a token; 16 bytes in the block of 576 threads (96 registers).
template <int kThreads>
constexpr int kBound = kThreads == 288 ? 320 : kThreads;
template <int kThreads, int kQAtOnce>
constexpr int kBlocks = kThreads != 288 ? 1 : kQAtOnce == 2 ? 3 : 2;

// D: dims of a query or key head (and of a value head, if there are any).  kThreads: a multiple of 32 and of D / 16.
template <typename T, int D, bool kE4M3, int kThreads, int kQAtOnce>
__global__ void __launch_bounds__(kBound<kThreads>, kBlocks<kThreads, kQAtOnce>) kv_append_kernel(KvAppendArgs a) {
  constexpr int kKvAtOnce = D == 576 ? 1 : 2;   // (a token has one latent row)
  constexpr int kPlaces = D / 16, kRows = kThreads / kPlaces;   // threads of a row, rows of a block at a time
  static_assert(kThreads % 32 == 0 && kThreads % kPlaces == 0, "whole rows");
  const int tid = threadIdx.x;
  const int64_t tok = blockIdx.x;
  // ---- the thread's place: vectors v0 and v1 (of eight elements) of every row it visits
  const int place = tid % kPlaces, row0 = tid / kPlaces;
  const bool turns = 16 * place < a.d_rope;
  int v0, v1;
  if (turns) {
    v0 = a.rope_at / 8 + (a.interleaved ? 2 * place : place);
    v1 = v0 + (a.interleaved ? 1 : a.d_rope / 16);
  } else {   // two neighbours of what is left (it starts and ends on a multiple of 16 dims)
    v0 = 2 * place - a.d_rope / 8;
    if (v0 >= a.rope_at / 8) v0 += a.d_rope / 8;
    v1 = v0 + 1;
  }
  const int e0 = 8 * v0, e1 = 8 * (v1 - v0);
  const int n_q = a.q != nullptr && (turns || a.q != a.q_out) ? a.H : 0;   // (what is not rotated in place stays)
  const int n_kv = a.latent ? a.G : 2 * a.G;                               // key rows, then value rows
  // (a row past the last is the last once more: no branches around loads; stores are guarded)
  auto q_row = [&](int r) -> const T* { return static_cast<const T*>(a.q) + tok * a.ld_q + min(r, a.H - 1) * D + e0; };
  auto kv_row = [&](int r) -> const T* {
    r = min(r, n_kv - 1);
    return (r < a.G ? static_cast<const T*>(a.k_new) + tok * a.ld_k_new + r * D : static_cast<const T*>(a.v_new) + tok * a.ld_v_new + (r - a.G) * D) + e0;
  };
  auto load = [&](const T* p, uint4 (&u)[2]) {
    u[0] = __ldcs(reinterpret_cast<const uint4*>(p));
    u[1] = __ldcs(reinterpret_cast<const uint4*>(p + e1));
  };
  uint4 uq[kQAtOnce][2], ukv[kKvAtOnce][2];
  pdl_wait();
  pdl_launch_dependents();
  // the rows do not depend on where they go: they are on their way while that is looked up
  if (n_q > 0) {
#pragma unroll
    for (int k = 0; k < kQAtOnce; ++k) load(q_row(row0 + k * kRows), uq[k]);
  }
#pragma unroll
  for (int k = 0; k < kKvAtOnce; ++k) load(kv_row(row0 + k * kRows), ukv[k]);

  // ---- the token's sequence, position and cache row (the same loads in every thread of the block)
  int b = static_cast<int>(tok);
  int64_t pos;
  bool mine = true;
  if (a.tok_start != nullptr) {
    int lo = 0, hi = a.batch;   // the last sequence that starts at or before the token
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.tok_start[mid] <= tok) lo = mid;
      else hi = mid;
    }
    b = lo;
    const int64_t t0 = a.tok_start[b];
    mine = tok >= t0 && tok < a.tok_start[b + 1];   // else padding
    pos = a.ctx_len[b] + (tok - t0);
  } else {
    pos = a.ctx_len[b];
  }
  const int64_t page_no = pos >> a.page_shift;
  bool fits = mine && pos >= 0 && a.ctx_len[b] >= 0 && page_no < a.pt_stride && (a.d_rope == 0 || pos < a.n_pos);
  int64_t row = 0;
  if (fits) {
    const int64_t page = a.page_table[b * a.pt_stride + page_no];
    fits = page >= 0 && page < a.n_pages;
    row = (page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
  }
  if (mine && !fits && tid == 0) paged::report_index(a.notice);

  if (fits) {
    float2 c[4], s[4];   // of the eight pairs
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      c[j] = make_float2(1.f, 1.f);
      s[j] = make_float2(0.f, 0.f);
    }
    if (turns) {
      const float* at = a.cos_sin + pos * a.d_rope + 8 * place;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 x = __ldg(reinterpret_cast<const float4*>(at) + h), y = __ldg(reinterpret_cast<const float4*>(at + a.d_rope / 2) + h);
        c[2 * h] = make_float2(x.x, x.y);
        c[2 * h + 1] = make_float2(x.z, x.w);
        s[2 * h] = make_float2(y.x, y.y);
        s[2 * h + 1] = make_float2(y.z, y.w);
      }
    }
    // x cos - y sin and y cos + x sin of the eight pairs of x[0 .. 15]
    auto turn = [&](float (&x)[16]) {
      if (a.interleaved) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = x[2 * j], q = x[2 * j + 1], cc = j & 1 ? c[j / 2].y : c[j / 2].x, ss = j & 1 ? s[j / 2].y : s[j / 2].x;
          x[2 * j] = p * cc - q * ss;
          x[2 * j + 1] = q * cc + p * ss;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 p = make_float2(x[2 * j], x[2 * j + 1]), q = make_float2(x[8 + 2 * j], x[8 + 2 * j + 1]);
          const float2 zero = make_float2(0.f, 0.f), minus = make_float2(-q.x, -q.y);
          const float2 u = fma2(p, c[j], fma2(minus, s[j], zero)), v = fma2(q, c[j], fma2(p, s[j], zero));
          x[2 * j] = u.x; x[2 * j + 1] = u.y;
          x[8 + 2 * j] = v.x; x[8 + 2 * j + 1] = v.y;
        }
      }
    };
    auto turned = [&](uint4 (&u)[2]) {
      float x[16];
      unpack8<T>(u[0], x);
      unpack8<T>(u[1], x + 8);
      turn(x);
      u[0] = pack8<T>(x);
      u[1] = pack8<T>(x + 8);
    };

    // ---- query heads
    T* q_out = static_cast<T*>(a.q_out) + tok * a.ld_q_out + e0;
    for (int r0 = row0; r0 < n_q; r0 += kQAtOnce * kRows) {
      if (r0 != row0) {
#pragma unroll
        for (int k = 0; k < kQAtOnce; ++k) load(q_row(r0 + k * kRows), uq[k]);
      }
#pragma unroll
      for (int k = 0; k < kQAtOnce; ++k) {
        const int r = r0 + k * kRows;
        if (turns) turned(uq[k]);
        if (r < n_q) {
          *reinterpret_cast<uint4*>(q_out + r * D) = uq[k][0];
          *reinterpret_cast<uint4*>(q_out + r * D + e1) = uq[k][1];
        }
      }
    }

    // ---- key heads, then value heads
    for (int r0 = 0; r0 < n_kv; r0 += kKvAtOnce * kRows) {   // (the same trips for all lanes of a warp: the shuffles below)
      if (r0 > 0) {
#pragma unroll
        for (int k = 0; k < kKvAtOnce; ++k) load(kv_row(r0 + row0 + k * kRows), ukv[k]);
      }
#pragma unroll
      for (int k = 0; k < kKvAtOnce; ++k) {
        const int r = r0 + row0 + k * kRows;
        const bool on = r < n_kv, is_v = r >= a.G;
        const int g = is_v ? r - a.G : r;
        const int64_t at = row * (is_v ? a.ld_v : a.ld_k) + g * D + e0;
        void* pool = is_v ? a.v_pool : a.k_pool;
        if constexpr (kE4M3) {
          float x[16];
          unpack8<T>(ukv[k][0], x);
          unpack8<T>(ukv[k][1], x + 8);
          if (turns && !is_v) turn(x);
          float top = 0.f;
#pragma unroll
          for (int j = 0; j < 16; ++j) top = fmaxf(top, fabsf(x[j]));
#pragma unroll
          for (int o = kPlaces / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          float scale = __fdiv_rn(top, 448.f);
          if (scale == 0.f) scale = 1.f;   // (a zero row, or one so small that the quotient is)
          const float inv = __frcp_rn(scale);
          const uint2 lo = codes8(x, scale, inv), hi = codes8(x + 8, scale, inv);
          if (on) {
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(pool) + at) = lo;
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(pool) + at + e1) = hi;
            if (place == 0) (is_v ? a.v_scale : a.k_scale)[row * a.G + g] = scale;
          }
        } else {
          if (turns && !is_v) turned(ukv[k]);
          if (on) {
            *reinterpret_cast<uint4*>(static_cast<T*>(pool) + at) = ukv[k][0];
            *reinterpret_cast<uint4*>(static_cast<T*>(pool) + at + e1) = ukv[k][1];
          }
        }
      }
    }
  }

  // ---- lengths.  One token per sequence: its block is the only one that reads its length, so the new one may take its place.
  if (a.ctx_len_out != nullptr) {
    if (a.tok_start == nullptr) {
      const int n = a.ctx_len[b];
      __syncthreads();
      if (tid == 0) a.ctx_len_out[b] = n + 1;
    } else if (tok == 0) {
      for (int i = tid; i < a.batch; i += blockDim.x) a.ctx_len_out[i] = new_length(a, i);
    }
  }
}

// New lengths where other blocks may still read the old ones, or where there are no tokens.
__global__ void kv_lengths_kernel(KvAppendArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < a.batch; i += gridDim.x * blockDim.x) a.ctx_len_out[i] = new_length(a, i);
}

template <typename T, int D, bool kE4M3>
cudaError_t launch_t(const KvAppendArgs& a, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>(a.n_tok));
  constexpr int kFew = kFewTokens<D>, kMany = kManyTokens<D>, kRows = kMany / (D / 16);   // rows of the smaller block at a time
  const int rows = std::max(a.q != nullptr ? a.H : 0, a.latent ? 1 : 2 * a.G);
  if (a.n_tok <= a.sm_count && rows > 4 * kRows) return launch_pdl(kv_append_kernel<T, D, kE4M3, kFew, 4>, grid, dim3(kFew), 0, st, a);
  if constexpr (D == 576)
    if (rows <= 2 * kRows) return launch_pdl(kv_append_kernel<T, D, kE4M3, kMany, 2>, grid, dim3(kMany), 0, st, a);
  return launch_pdl(kv_append_kernel<T, D, kE4M3, kMany, 4>, grid, dim3(kMany), 0, st, a);
}
template <typename T>
cudaError_t launch_d(const KvAppendArgs& a, cudaStream_t st) {
  if (a.d == 576) return launch_t<T, 576, false>(a, st);
  if (a.d == 128) return a.e4m3 ? launch_t<T, 128, true>(a, st) : launch_t<T, 128, false>(a, st);
  return a.e4m3 ? launch_t<T, 64, true>(a, st) : launch_t<T, 64, false>(a, st);
}

}  // namespace

cudaError_t launch_kv_append(const KvAppendArgs& args, cudaStream_t st, int64_t* n_launch) {
  KvAppendArgs a = args;
  // with several tokens a sequence its length is read by several blocks
  const bool later = a.tok_start != nullptr && a.ctx_len_out != nullptr && (a.n_tok == 0 || a.ctx_len_out == a.ctx_len);
  if (later) a.ctx_len_out = nullptr;
  cudaError_t e = cudaSuccess;
  if (a.n_tok > 0) {
    e = a.fp16 ? launch_d<__half>(a, st) : launch_d<__nv_bfloat16>(a, st);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    ++*n_launch;
  }
  if (later) {
    a.ctx_len_out = args.ctx_len_out;
    e = launch_pdl(kv_lengths_kernel, dim3((a.batch + 255) / 256), dim3(256), 0, st, a);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e == cudaSuccess) ++*n_launch;
  }
  return e;
}

}  // namespace lsa
