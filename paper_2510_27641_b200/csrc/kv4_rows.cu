// specattn_kv4_append, specattn_kv4_read: rows of 128 values in and out of a cache that holds them in 4 bits.
//
// Both are copies that change a row's size (256 bytes <-> 68), bound by HBM for prompts and by the chain start ->
// block table -> row for the few tokens of a step.  A row belongs to half a warp, 16 bytes of values to a lane: the
// row's minimum and maximum are four exchanges between lanes, and both sides of the copy are whole sectors.  A
// half-warp has kRows rows in flight, whose loads are sent before the page of any is known.
#include <cuda_runtime.h>
#include <float.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "kv4.cuh"
#include "nvtx_range.h"

namespace specattn {

extern std::atomic<long long> g_launch_count;

namespace {

constexpr int kThreads = 256;
constexpr int kHalfWarps = kThreads / 16;
constexpr int kRows = 4;

struct RowsParams {
  Kv4View cache;
  unsigned char *k, *v;
  long long k_batch, k_token, k_head, v_batch, v_token, v_head;  // bytes
  const int *start, *n_new;
  int* status;
  int n_tokens, heads, batch;
  int heads_first;  // which of two neighbouring rows of a block share a token (1) or a head (0)
};

// The min(15, rint(d / s)) of the cache's definition, d / s being the correctly rounded quotient.  A product with
// 1/s decides it except within 1e-5 of a border between two codes (its error is below 3e-6 for quotients up to 16);
// 16-bit values meet borders exactly, so that case is real and divides.
__device__ __forceinline__ uint32_t code_of(float d, float s, float inv) {
  const float q = d * inv;
  float c = rintf(q);
  if (fabsf(fabsf(q - c) - 0.5f) < 1e-5f) c = rintf(__fdiv_rn(d, s));
  return static_cast<uint32_t>(fminf(c, 15.f));
}

// A block takes `per_block` rows of one sequence: rows are numbered (token, side, head) with heads or tokens
// innermost, as they lie closer together in the cache.
template <bool kHalf, bool kAppend>
__global__ void __launch_bounds__(kThreads) kv4_rows_kernel(const __grid_constant__ RowsParams P, int tokens_per_block) {
  const int b = blockIdx.y, lane = threadIdx.x & 15, hw = threadIdx.x >> 4;
  const int t0 = blockIdx.x * tokens_per_block;
  int n = P.n_tokens;
  if (P.n_new != nullptr) n = min(n, max(0, P.n_new[b]));
  const int n_t = min(tokens_per_block, n - t0);
  if (n_t <= 0) return;
  const long long first = P.start[b];
  const int rows = n_t * 2 * P.heads;
  const uint32_t mask = 0xffffu << (threadIdx.x & 16);
  for (int r0 = hw; r0 < rows; r0 += kHalfWarps * kRows) {
    int t[kRows], kv[kRows], head[kRows];
    unsigned char* at[kRows];
    uint4 x[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      const int r = r0 + j * kHalfWarps;
      const int in = P.heads_first ? P.heads : n_t, out = r / in;
      head[j] = P.heads_first ? r - out * in : out >> 1;
      t[j] = t0 + (P.heads_first ? out >> 1 : r - out * in);
      kv[j] = out & 1;
      at[j] = (kv[j] ? P.v + b * P.v_batch + t[j] * P.v_token + head[j] * P.v_head
                     : P.k + b * P.k_batch + t[j] * P.k_token + head[j] * P.k_head) + lane * 16;
      if (kAppend && r < rows) x[j] = __ldcs(reinterpret_cast<const uint4*>(at[j]));
    }
    unsigned char *codes[kRows], *params[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      codes[j] = params[j] = nullptr;
      if (r0 + j * kHalfWarps >= rows) continue;
      const long long pos = first + t[j], pi = pos < 0 ? -1 : pos / P.cache.page_size;
      const long long page = page_of(P.cache.table, P.cache.table_stride, P.cache.n_pages, b, pi);
      if (page < 0) {
        if (P.status != nullptr && lane == 0) atomicOr(P.status + b, SPECATTN_ROW_BAD_INDEX);
        continue;
      }
      const long long slot = pos - pi * P.cache.page_size;
      codes[j] = P.cache.codes + page * P.cache.s_page + kv[j] * P.cache.s_kv + slot * P.cache.s_slot + head[j] * P.cache.s_head + lane * 4;
      params[j] = P.cache.params + page * P.cache.p_page + kv[j] * P.cache.p_kv + slot * P.cache.p_slot + head[j] * P.cache.p_head;
    }
    if (kAppend) {
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        if (r0 + j * kHalfWarps >= rows) break;  // (the same for the whole half-warp)
        float f[8];
        const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 p = widen<kHalf>(w[i]);
          f[2 * i] = p.x;
          f[2 * i + 1] = p.y;
        }
        float lo = f[0], hi = f[0], nan = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          lo = fminf(lo, f[i]);
          hi = fmaxf(hi, f[i]);
          nan = fmaf(f[i], 0.f, nan);  // 0 unless a value is NaN or infinite
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
          lo = fminf(lo, __shfl_xor_sync(mask, lo, o));
          hi = fmaxf(hi, __shfl_xor_sync(mask, hi, o));
          nan += __shfl_xor_sync(mask, nan, o);
        }
        const float span = __fsub_rn(hi, lo);
        const bool fine = nan == 0.f && span <= FLT_MAX;
        const uint32_t s16 = narrow<kHalf>(__fdiv_rn(span, 15.f), lo);
        float s = widen<kHalf>(s16).x;
        const bool usable = fine && s >= FLT_MIN;
        if (!usable) s = 1.f;
        const float inv = __fdiv_rn(1.f, s);
        uint32_t c = 0;
        if (usable) {
#pragma unroll
          for (int i = 0; i < 8; ++i) c |= code_of(__fsub_rn(f[i], lo), s, inv) << (4 * i);
        }
        if (codes[j] != nullptr) {
          *reinterpret_cast<uint32_t*>(codes[j]) = c;
          if (lane == 0) {
            const uint32_t nan16 = kHalf ? 0x7e007e00u : 0x7fc07fc0u;
            *reinterpret_cast<uint32_t*>(params[j]) = !fine ? nan16 : usable ? s16 : (s16 & 0xffff0000u);
            if (!fine && P.status != nullptr) atomicOr(P.status + b, SPECATTN_ROW_INVALID_VALUE);
          }
        }
      }
    } else {
      uint32_t c[kRows], sz[kRows];
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        if (codes[j] == nullptr) continue;
        c[j] = __ldg(reinterpret_cast<const uint32_t*>(codes[j]));
        sz[j] = __ldg(reinterpret_cast<const uint32_t*>(params[j]));
      }
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        if (codes[j] == nullptr) continue;
        const float2 p = widen<kHalf>(sz[j]);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // (a product of 11 by 4 bits is exact, so the fused form rounds once like the separate one)
          const float lo = fmaf(p.x, static_cast<float>((c[j] >> (8 * i)) & 15u), p.y);
          const float hi = fmaf(p.x, static_cast<float>((c[j] >> (8 * i + 4)) & 15u), p.y);
          w[i] = narrow<kHalf>(lo, hi);
        }
        __stcs(reinterpret_cast<uint4*>(at[j]), make_uint4(w[0], w[1], w[2], w[3]));
      }
    }
  }
}

int rows_call(const specattn_kv4_rows_args* args, void* cuda_stream, bool append) {
  if (args == nullptr) return SPECATTN_ERR_NULL;
  if (args->struct_size != sizeof(specattn_kv4_rows_args)) return SPECATTN_ERR_STRUCT_SIZE;
  const specattn_kv4_rows_args& A = *args;
  if (A.batch < 0 || A.batch > 65535 || A.n_tokens < 0 || A.n_kv_heads < 1 || A.n_kv_heads > 65535 || A.reserved != 0)
    return SPECATTN_ERR_RANGE;
  const int cc = kv4_check(A.cache);
  if (cc != SPECATTN_OK) return cc;
  if (A.head_dim != kKv4D) return SPECATTN_ERR_UNSUPPORTED;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (A.batch == 0) return SPECATTN_OK;
  if (!A.k || !A.v || !A.start) return SPECATTN_ERR_NULL;
  const int cb = kv4_check_buffers(A.cache);
  if (cb != SPECATTN_OK) return cb;
  if (reinterpret_cast<uintptr_t>(A.k) % 16 != 0 || reinterpret_cast<uintptr_t>(A.v) % 16 != 0) return SPECATTN_ERR_ALIGN;
  if (A.k_stride_batch % 8 || A.k_stride_token % 8 || A.k_stride_head % 8 || A.v_stride_batch % 8 || A.v_stride_token % 8 ||
      A.v_stride_head % 8)
    return SPECATTN_ERR_ALIGN;
  if (A.status != nullptr &&
      cudaMemsetAsync(A.status, 0, static_cast<size_t>(A.batch) * sizeof(int32_t), stream) != cudaSuccess) {
    cudaGetLastError();
    return SPECATTN_ERR_CUDA;
  }
  if (A.n_tokens == 0) return SPECATTN_OK;
  RowsParams P;
  P.cache = kv4_view(A.cache);
  P.k = static_cast<unsigned char*>(A.k);
  P.v = static_cast<unsigned char*>(A.v);
  P.k_batch = A.k_stride_batch * 2;
  P.k_token = A.k_stride_token * 2;
  P.k_head = A.k_stride_head * 2;
  P.v_batch = A.v_stride_batch * 2;
  P.v_token = A.v_stride_token * 2;
  P.v_head = A.v_stride_head * 2;
  P.start = A.start;
  P.n_new = A.n_new;
  P.status = A.status;
  P.n_tokens = A.n_tokens;
  P.heads = A.n_kv_heads;
  P.batch = A.batch;
  P.heads_first = llabs(A.cache.stride_head) < llabs(A.cache.stride_slot) ? 1 : 0;
  // as many tokens to a block as give its half-warps kRows rows each
  int per_block = kHalfWarps * kRows / (2 * A.n_kv_heads);
  if (per_block < 1) per_block = 1;
  const dim3 grid((A.n_tokens + per_block - 1) / per_block, A.batch);
  const bool half = A.cache.dtype == SPECATTN_DTYPE_FP16;
  if (append) {
    if (half)
      kv4_rows_kernel<true, true><<<grid, kThreads, 0, stream>>>(P, per_block);
    else
      kv4_rows_kernel<false, true><<<grid, kThreads, 0, stream>>>(P, per_block);
  } else {
    if (half)
      kv4_rows_kernel<true, false><<<grid, kThreads, 0, stream>>>(P, per_block);
    else
      kv4_rows_kernel<false, false><<<grid, kThreads, 0, stream>>>(P, per_block);
  }
  if (cudaGetLastError() != cudaSuccess) return SPECATTN_ERR_CUDA;
  g_launch_count.fetch_add(1, std::memory_order_relaxed);
  return SPECATTN_OK;
}

}  // namespace
}  // namespace specattn

extern "C" int specattn_kv4_append(const specattn_kv4_rows_args* args, void* cuda_stream) {
  specattn::NvtxRange nvtx_range("specattn_kv4_append");
  return specattn::rows_call(args, cuda_stream, true);
}

extern "C" int specattn_kv4_read(const specattn_kv4_rows_args* args, void* cuda_stream) {
  specattn::NvtxRange nvtx_range("specattn_kv4_read");
  return specattn::rows_call(args, cuda_stream, false);
}
