// specattn_kv4_append, specattn_kv4_read: rows of 128 values in and out of a cache that holds them in 4 bits.
//
// Both are copies that change a row's size (256 bytes <-> 68), bound by HBM and, on the way in, nearly as much by
// instructions for prompts (437k rows: 45 us in, 30 back; 3.2 and 4.7 TB/s), and by the chain start -> block table -> row
// for the few tokens of a step (4 to 5 us each).  A row belongs to half a warp, 16 bytes of values to a lane: both
// sides of the copy are whole sectors.  A half-warp has kRows rows in flight, whose values are asked for before the page
// of any is known, and finds their minima and maxima together.
#include <cuda_runtime.h>
#include <float.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "kv4.cuh"
#include "nvtx_range.h"

namespace specattn {

extern std::atomic<long long> g_launch_count;
int device_sm_count();

namespace {

constexpr int kThreads = 256;
constexpr int kHalfWarps = kThreads / 16;
constexpr int kRows = 8;

struct RowsParams {
  Kv4View cache;
  unsigned char *k, *v;
  long long k_batch, k_token, k_head, v_batch, v_token, v_head;  // bytes
  const int *start, *n_new;
  int* status;
  int n_tokens, heads, batch;
  FastDiv by_heads;
  int heads_first;  // which of two neighbouring rows of a block share a token (1) or a head (0)
};

// A pair of 16-bit values by pair: the smaller and the larger ones, NaN where either is.
template <bool kHalf>
__device__ __forceinline__ uint32_t least(uint32_t a, uint32_t b) {
  if (kHalf) {
    const __half2 v = __hmin2_nan(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  const __nv_bfloat162 v = __hmin2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <bool kHalf>
__device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) {
  if (kHalf) {
    const __half2 v = __hmax2_nan(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  const __nv_bfloat162 v = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}

constexpr float kRound = 12582912.f;  // 1.5 2^23: a number of less than 2^22 added to it is rounded to an integer, to even

// The smallest / largest of the 16 lanes' values of eight rows: lane l gets those of row l & 7.  Three exchanges halve the rows
// that a lane still answers for (4 + 2 + 1 shuffles), one more joins the two lanes of a row: a quarter of the shuffles
// of eight separate reductions.
template <typename Op>
__device__ __forceinline__ uint32_t of_eight_rows(uint32_t (&x)[kRows], int lane, uint32_t mask, Op op) {
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) {
    const bool upper = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const uint32_t keep = upper ? x[i + o] : x[i], give = upper ? x[i] : x[i + o];
      x[i] = op(keep, __shfl_xor_sync(mask, give, o));
    }
  }
  return op(x[0], __shfl_xor_sync(mask, x[0], 8));
}

// The codes of eight values, packed:  min(15, rint(d / s)), d / s being the correctly rounded quotient.  A product with
// 1/s decides it except within 1e-5 of a border between two codes (it is off by less than 3e-6 for quotients up to
// 16); 16-bit values meet borders exactly, so that case is real and divides.  So do rows whose scale is subnormal
// in fp16, which alone can have quotients of 15.5 and more.
template <bool kHalf>
__device__ __forceinline__ uint32_t encode(const uint4& x, float lo, float inv) {
  if (inv == 0.f) return 0;  // (a constant row, or none of finite span)
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  float c[8], far = kHalf && inv > 16384.f ? 1.f : 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = widen<kHalf>(w[i]);
    const Two q = mul2(add2(two(p.x, p.y), two(-lo, -lo)), two(inv, inv));
    const Two r = add2(add2(q, two(kRound, kRound)), two(-kRound, -kRound));
    const float2 off = each(fma2(r, two(-1.f, -1.f), q)), code = each(r);
    c[2 * i] = code.x, c[2 * i + 1] = code.y;
    far = fmaxf(far, fmaxf(fabsf(off.x), fabsf(off.y)));
  }
  if (far > 0.49999f) {
    // the scale, which is a 16-bit value, back from its rounded inverse
    const float s = widen<kHalf>(narrow<kHalf>(__fdiv_rn(1.f, inv), 0.f)).x;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 p = widen<kHalf>(w[i >> 1]);
      c[i] = fminf(rintf(__fdiv_rn(__fsub_rn(i & 1 ? p.y : p.x, lo), s)), 15.f);
    }
  }
  // four codes are a number below 2^16, exact in binary32
  const float a = fmaf(fmaf(c[3], 16.f, c[2]), 256.f, fmaf(c[1], 16.f, c[0]));
  const float b = fmaf(fmaf(c[7], 16.f, c[6]), 256.f, fmaf(c[5], 16.f, c[4]));
  return __byte_perm(__float_as_uint(__fadd_rn(a, 8388608.f)), __float_as_uint(__fadd_rn(b, 8388608.f)), 0x5410);
}

// A block takes the rows of up to tokens_per_block tokens of one sequence, eight consecutive ones to a half-warp at a
// time: rows are numbered (token, side, head) with heads or tokens innermost, as they lie closer together in the
// cache.  Lane l of the sixteen finds out where row l & 7 lies, and what its scale is; the others ask it.
template <bool kHalf, bool kAppend>
__global__ void __launch_bounds__(kThreads, 4) kv4_rows_kernel(const __grid_constant__ RowsParams P, int tokens_per_block) {
  const int b = blockIdx.y, lane = threadIdx.x & 15, hw = threadIdx.x >> 4, own = lane & (kRows - 1);
  const int t0 = blockIdx.x * tokens_per_block;
  int n = P.n_tokens;
  if (P.n_new != nullptr) n = min(n, max(0, P.n_new[b]));
  const int n_t = min(tokens_per_block, n - t0);
  if (n_t <= 0) return;
  const long long first = P.start[b];
  const int rows = n_t * 2 * P.heads;
  const uint32_t mask = 0xffffu << (threadIdx.x & 16);
  for (int r0 = hw * kRows; r0 < rows; r0 += kHalfWarps * kRows) {
    const int r = r0 + own;
    unsigned char* at = nullptr;  // of the values
    long long code_at = -1;       // of the codes, from the cache's first; -1: nowhere
    unsigned char* param_at = nullptr;
    if (r < rows) {
      const int out = P.heads_first ? r / P.by_heads : r / n_t;
      const int head = P.heads_first ? r - out * P.heads : out >> 1, kv = out & 1;
      const int t = t0 + (P.heads_first ? out >> 1 : r - out * n_t);
      at = (kv ? P.v : P.k) + b * (kv ? P.v_batch : P.k_batch) + t * (kv ? P.v_token : P.k_token) + head * (kv ? P.v_head : P.k_head);
      const long long pos = first + t;
      long long page = -1;
      int slot = 0;
      if (pos >= 0 && pos <= INT32_MAX) {
        const int pi = static_cast<int>(pos) / P.cache.by_page;
        page = page_of(P.cache.table, P.cache.table_stride, P.cache.n_pages, b, pi);
        slot = static_cast<int>(pos) - pi * P.cache.page_size;
      }
      if (page >= 0) {
        code_at = reinterpret_cast<long long>(P.cache.codes) + page * P.cache.s_page + kv * P.cache.s_kv + slot * P.cache.s_slot + head * P.cache.s_head;
        param_at = P.cache.params + page * P.cache.p_page + kv * P.cache.p_kv + slot * P.cache.p_slot + head * P.cache.p_head;
      } else if (P.status != nullptr && lane < kRows) {
        atomicOr(P.status + b, SPECATTN_ROW_BAD_INDEX);
      }
    }
    if (kAppend) {
      uint4 x[kRows];
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        const unsigned long long from = __shfl_sync(mask, reinterpret_cast<unsigned long long>(at), j, 16);
        x[j] = make_uint4(0u, 0u, 0u, 0u);
        if (from != 0) x[j] = __ldcs(reinterpret_cast<const uint4*>(from + lane * 16));
      }
      uint32_t small[kRows], large[kRows];
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        small[j] = least<kHalf>(least<kHalf>(x[j].x, x[j].y), least<kHalf>(x[j].z, x[j].w));
        large[j] = most<kHalf>(most<kHalf>(x[j].x, x[j].y), most<kHalf>(x[j].z, x[j].w));
      }
      uint32_t lo2 = of_eight_rows(small, lane, mask, least<kHalf>), hi2 = of_eight_rows(large, lane, mask, most<kHalf>);
      lo2 = least<kHalf>(lo2, __byte_perm(lo2, 0, 0x1032));
      hi2 = most<kHalf>(hi2, __byte_perm(hi2, 0, 0x1032));
      const float lo = widen<kHalf>(lo2).x, span = __fsub_rn(widen<kHalf>(hi2).x, lo);
      const bool fine = span <= FLT_MAX;  // (false for NaN, which the smallest and largest pass on)
      const uint32_t s16 = narrow<kHalf>(__fdiv_rn(span, 15.f), lo);
      const float s = widen<kHalf>(s16).x;
      const bool usable = fine && s >= FLT_MIN;
      const float inv = usable ? __fdiv_rn(1.f, s) : 0.f;
      if (code_at >= 0 && lane < kRows) {
        *reinterpret_cast<uint32_t*>(param_at) = !fine ? (kHalf ? 0x7e007e00u : 0x7fc07fc0u) : usable ? s16 : (s16 & 0xffff0000u);
        if (!fine && P.status != nullptr) atomicOr(P.status + b, SPECATTN_ROW_INVALID_VALUE);
      }
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        const long long to = __shfl_sync(mask, code_at, j, 16);
        const float lo_j = __shfl_sync(mask, lo, j, 16), inv_j = __shfl_sync(mask, inv, j, 16);
        if (to >= 0) *reinterpret_cast<uint32_t*>(to + lane * 4) = encode<kHalf>(x[j], lo_j, inv_j);
      }
    } else {
      const uint32_t sz = code_at >= 0 ? __ldcs(reinterpret_cast<const uint32_t*>(param_at)) : 0u;
      uint32_t c[kRows];
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        const long long from = __shfl_sync(mask, code_at, j, 16);
        c[j] = from >= 0 ? __ldcs(reinterpret_cast<const uint32_t*>(from + lane * 4)) : 0u;
      }
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        const unsigned long long into = __shfl_sync(mask, code_at >= 0 ? reinterpret_cast<unsigned long long>(at) : 0ull, j, 16);
        const float2 p = widen<kHalf>(__shfl_sync(mask, sz, j, 16));
        const uint32_t low = c[j] & 0x0f0f0f0fu, high = (c[j] >> 4) & 0x0f0f0f0fu;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // (a code in the lowest byte of 2^23 makes 2^23 and that number; a product of 11 by 4 bits is exact, so the fused
          // form rounds once like the separate one)
          const float a = __uint_as_float(__byte_perm(low, 0x4b000000u, 0x7650 + i)),
                      b = __uint_as_float(__byte_perm(high, 0x4b000000u, 0x7650 + i));
          const float2 x = each(fma2(two(p.x, p.x), add2(two(a, b), two(-8388608.f, -8388608.f)), two(p.y, p.y)));
          w[i] = narrow<kHalf>(x.x, x.y);
        }
        if (into != 0) __stcs(reinterpret_cast<uint4*>(into + lane * 16), make_uint4(w[0], w[1], w[2], w[3]));
      }
    }
  }
}

int rows_call(const specattn_kv4_rows_args* args, void* cuda_stream, bool append) {
  if (args == nullptr) return SPECATTN_ERR_NULL;
  if (args->struct_size != sizeof(specattn_kv4_rows_args)) return SPECATTN_ERR_STRUCT_SIZE;
  const specattn_kv4_rows_args& A = *args;
  if (A.batch < 0 || A.batch > 65535 || A.n_tokens < 0 || A.n_kv_heads < 1 || A.n_kv_heads > 65535 || A.cache.n_pages > INT32_MAX || A.reserved != 0)
    return SPECATTN_ERR_RANGE;
  const int cc = kv4_check(A.cache);
  if (cc != SPECATTN_OK) return cc;
  if (A.head_dim != kKv4D) return SPECATTN_ERR_UNSUPPORTED;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (A.batch == 0) return SPECATTN_OK;
  if ((A.n_tokens > 0 && (!A.k || !A.v)) || !A.start) return SPECATTN_ERR_NULL;
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
  const int sms = device_sm_count();
  if (sms <= 0) return SPECATTN_ERR_CUDA;
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
  P.by_heads = fast_div(A.n_kv_heads);
  P.batch = A.batch;
  P.heads_first = llabs(A.cache.stride_head) < llabs(A.cache.stride_slot) ? 1 : 0;
  // as many tokens to a block as give its half-warps kRows rows each
  int per_block = kHalfWarps * kRows / (2 * A.n_kv_heads);
  // (a few tokens are spread over more blocks: latency is all there is to them)
  while (per_block > 1 && static_cast<long long>(A.batch) * (((A.n_tokens - 1) / per_block + 1)) < sms) per_block = (per_block + 1) / 2;
  if (per_block < 1) per_block = 1;
  const dim3 grid((A.n_tokens - 1) / per_block + 1, A.batch);
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
