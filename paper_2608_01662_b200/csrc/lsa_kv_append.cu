// lsa_kv_append: new tokens of a batch of sequences into the rows of a paged cache.
//
// A block takes one token: its query heads, key heads and value heads are rows of D elements.  A thread keeps one place
// within a row for all rows that it visits: 16 dims, two 16-byte vectors.  In the rotated part these are the two halves of
// eight pairs (x cos - y sin, y cos + x sin), so the angles' cosines and sines are fetched once per thread, not once per head; a
// row's threads are consecutive lanes, so the largest element of an e4m3 row is a few shuffles.
//
// Bound: HBM for prompts (read and write once), a launch and the chain length -> page -> row for decode steps.
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
// Eight codes of value / scale: round to nearest even, saturating.
__device__ __forceinline__ uint2 codes8(const float* x, float scale) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t r = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float2 v = make_float2(__fdiv_rn(x[4 * h + 2 * j], scale), __fdiv_rn(x[4 * h + 2 * j + 1], scale));
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

constexpr int kRowsInFlight = 4;
// Threads of a block: few tokens get a block that has all rows of 64 heads of 576 dims in flight at once; of many tokens several
// share an SM.
template <int D>
constexpr int kFewTokens = D == 576 ? 576 : 512;
template <int D>
constexpr int kManyTokens = D == 576 ? 288 : 64;

// D: dims of a query or key head (and of a value head, if there are any).  Blocks are a multiple of 32 and of D / 16 threads.
template <typename T, int D, bool kE4M3>
__global__ void __launch_bounds__(kFewTokens<D>) kv_append_kernel(KvAppendArgs a) {
  constexpr int kPlaces = D / 16;   // threads of a row
  const int tid = threadIdx.x;
  const int64_t tok = blockIdx.x;
  // ---- the thread's place: vectors v0 and v1 (of eight elements) of every row it visits
  const int place = tid % kPlaces, lane_row = tid / kPlaces, rows_at_once = blockDim.x / kPlaces;
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
  // rows of the token: query heads, key heads, value heads
  const int n_q = a.q != nullptr ? a.H : 0, n_k = n_q + a.G, n_rows = a.latent ? n_k : n_k + a.G;
  const bool in_place = a.q == a.q_out;
  auto skipped = [&](int r) { return r >= n_rows || (r < n_q && in_place && !turns); };   // (what is not rotated in place stays)
  uint4 u[kRowsInFlight][2];
  auto fetch = [&](int r0) {
#pragma unroll
    for (int k = 0; k < kRowsInFlight; ++k) {
      const int r = r0 + k * rows_at_once + lane_row;
      if (skipped(r)) continue;
      const T* src = r < n_q ? static_cast<const T*>(a.q) + tok * a.ld_q + r * D
                     : r < n_k ? static_cast<const T*>(a.k_new) + tok * a.ld_k_new + (r - n_q) * D
                               : static_cast<const T*>(a.v_new) + tok * a.ld_v_new + (r - n_k) * D;
      u[k][0] = __ldcs(reinterpret_cast<const uint4*>(src + 8 * v0));
      u[k][1] = __ldcs(reinterpret_cast<const uint4*>(src + 8 * v1));
    }
  };
  pdl_wait();
  pdl_launch_dependents();
  fetch(0);   // the rows do not depend on where they go: they are on their way while that is looked up

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
    float c[8], s[8];
    if (turns) {
      const float4* cs = reinterpret_cast<const float4*>(a.cos_sin + pos * a.d_rope + 8 * place);
      const float4* sn = reinterpret_cast<const float4*>(a.cos_sin + pos * a.d_rope + a.d_rope / 2 + 8 * place);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 x = __ldg(cs + h), y = __ldg(sn + h);
        c[4 * h] = x.x; c[4 * h + 1] = x.y; c[4 * h + 2] = x.z; c[4 * h + 3] = x.w;
        s[4 * h] = y.x; s[4 * h + 1] = y.y; s[4 * h + 2] = y.z; s[4 * h + 3] = y.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = 1.f, s[j] = 0.f;
    }
    auto turn = [&](float (&x)[16]) {
      if (a.interleaved) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = x[2 * j], q = x[2 * j + 1];
          x[2 * j] = p * c[j] - q * s[j];
          x[2 * j + 1] = q * c[j] + p * s[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = x[j], q = x[j + 8];
          x[j] = p * c[j] - q * s[j];
          x[j + 8] = q * c[j] + p * s[j];
        }
      }
    };
    for (int r0 = 0; r0 < n_rows; r0 += kRowsInFlight * rows_at_once) {   // (the same trips for all lanes of a warp: the shuffles below)
      if (r0 > 0) fetch(r0);
#pragma unroll
      for (int k = 0; k < kRowsInFlight; ++k) {
        const int r = r0 + k * rows_at_once + lane_row;
        const bool on = !skipped(r), is_q = r < n_q, is_v = r >= n_k;
        float x[16];
        if (turns || kE4M3) {
          unpack8<T>(u[k][0], x);
          unpack8<T>(u[k][1], x + 8);
          if (turns && !is_v) turn(x);
        }
        if (kE4M3 && r0 + (k + 1) * rows_at_once > n_q) {   // block-uniform: rows of the cache are among these
          float top = 0.f;
#pragma unroll
          for (int j = 0; j < 16; ++j) top = fmaxf(top, fabsf(x[j]));
#pragma unroll
          for (int o = kPlaces / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          if (on && !is_q) {
            float scale = __fdiv_rn(top, 448.f);
            if (scale == 0.f) scale = 1.f;   // (a zero row, or one so small that the quotient is)
            const int g = is_v ? r - n_k : r - n_q;
            uint8_t* dst = static_cast<uint8_t*>(is_v ? a.v_pool : a.k_pool) + row * (is_v ? a.ld_v : a.ld_k) + g * D;
            *reinterpret_cast<uint2*>(dst + 8 * v0) = codes8(x, scale);
            *reinterpret_cast<uint2*>(dst + 8 * v1) = codes8(x + 8, scale);
            if (place == 0) (is_v ? a.v_scale : a.k_scale)[row * a.G + g] = scale;
          }
        }
        if (on && (is_q || !kE4M3)) {
          if (turns && !is_v) {
            u[k][0] = pack8<T>(x);
            u[k][1] = pack8<T>(x + 8);
          }
          T* dst = is_q ? static_cast<T*>(a.q_out) + tok * a.ld_q_out + r * D
                   : is_v ? static_cast<T*>(a.v_pool) + row * a.ld_v + (r - n_k) * D
                          : static_cast<T*>(a.k_pool) + row * a.ld_k + (r - n_q) * D;
          *reinterpret_cast<uint4*>(dst + 8 * v0) = u[k][0];
          *reinterpret_cast<uint4*>(dst + 8 * v1) = u[k][1];
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
  const int threads = a.n_tok <= 2 * a.sm_count ? kFewTokens<D> : kManyTokens<D>;
  return launch_pdl(kv_append_kernel<T, D, kE4M3>, dim3(static_cast<unsigned>(a.n_tok)), dim3(threads), 0, st, a);
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
  const uintptr_t in = reinterpret_cast<uintptr_t>(a.ctx_len), out = reinterpret_cast<uintptr_t>(a.ctx_len_out), bytes = static_cast<uintptr_t>(a.batch) * 4;
  const bool later = a.tok_start != nullptr && a.ctx_len_out != nullptr && (a.n_tok == 0 || (in < out + bytes && out < in + bytes));
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
