// What the kernels of the 4-bit cache share: the cache as a kernel sees it, the checks of the host side.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "specattn.h"

namespace specattn {

constexpr int kKv4D = 128;         // values of a row
constexpr int kKv4Row = kKv4D / 2;  // bytes of its codes

// Division of 0 <= n < 2^31 by a number that the host knows: n / d = (n m) >> s with m = ceil(2^s / d),
// s = 31 + ceil(log2 d), which is exact for these n because m d exceeds 2^s by less than 2^(s - 31).
struct FastDiv {
  unsigned m;
  int s;
};
inline FastDiv fast_div(int d) {
  int up = 0;
  while ((1ll << up) < d) ++up;
  FastDiv f;
  f.s = 31 + up;
  f.m = static_cast<unsigned>(((1ull << f.s) + d - 1) / d);
  return f;
}
__device__ __forceinline__ int operator/(int n, const FastDiv& f) {
  return static_cast<int>((static_cast<unsigned long long>(static_cast<unsigned>(n)) * f.m) >> f.s);
}

struct Kv4View {
  unsigned char* codes;
  unsigned char* params;  // pairs of 16-bit values, addressed in bytes here
  long long n_pages;
  long long s_page, s_kv, s_slot, s_head;  // bytes
  long long p_page, p_kv, p_slot, p_head;  // bytes
  const int* table;
  long long table_stride;
  int page_size;
  FastDiv by_page;
};

inline Kv4View kv4_view(const specattn_kv4_cache& c) {
  Kv4View v;
  v.codes = static_cast<unsigned char*>(c.codes);
  v.params = static_cast<unsigned char*>(c.params);
  v.n_pages = c.n_pages;
  v.s_page = c.stride_page;
  v.s_kv = c.stride_kv;
  v.s_slot = c.stride_slot;
  v.s_head = c.stride_head;
  v.p_page = c.pstride_page * 2;
  v.p_kv = c.pstride_kv * 2;
  v.p_slot = c.pstride_slot * 2;
  v.p_head = c.pstride_head * 2;
  v.table = c.block_table;
  v.table_stride = c.block_table_stride;
  v.page_size = c.page_size;
  v.by_page = fast_div(c.page_size);
  return v;
}

inline int kv4_check(const specattn_kv4_cache& c) {
  if (c.page_size < 1 || c.n_pages < 1 || c.block_table_stride < 0) return SPECATTN_ERR_RANGE;
  if (c.dtype != SPECATTN_DTYPE_BF16 && c.dtype != SPECATTN_DTYPE_FP16) return SPECATTN_ERR_RANGE;
  return SPECATTN_OK;
}

inline int kv4_check_buffers(const specattn_kv4_cache& c) {
  if (!c.codes || !c.params) return SPECATTN_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(c.codes) % 16 != 0 || reinterpret_cast<uintptr_t>(c.params) % 4 != 0)
    return SPECATTN_ERR_ALIGN;
  if (c.stride_page % 16 || c.stride_kv % 16 || c.stride_slot % 16 || c.stride_head % 16) return SPECATTN_ERR_ALIGN;
  if (c.pstride_page % 2 || c.pstride_kv % 2 || c.pstride_slot % 2 || c.pstride_head % 2) return SPECATTN_ERR_ALIGN;
  return SPECATTN_OK;
}

// The page of the page_index-th page of sequence b; -1 where there is none.
__device__ __forceinline__ long long page_of(const int* table, long long table_stride, long long n_pages, int b,
                                             int page_index) {
  if (page_index < 0 || page_index >= table_stride) return -1;
  const long long at = static_cast<long long>(b) * table_stride + page_index;
  const long long page = table != nullptr ? static_cast<long long>(table[at]) : at;
  return page >= 0 && page < n_pages ? page : -1;
}

// 16-bit values as binary32 and back (bf16 or fp16, to the nearest, ties to even).
template <bool kHalf>
__device__ __forceinline__ float2 widen(uint32_t pair) {
  if (kHalf) return __half22float2(*reinterpret_cast<const __half2*>(&pair));
  return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&pair));
}
template <bool kHalf>
__device__ __forceinline__ uint32_t narrow(float lo, float hi) {
  if (kHalf) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Two binary32 operations in one instruction.
struct Two {
  unsigned long long v;
};
__device__ __forceinline__ Two two(float a, float b) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 each(Two a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
  return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

}  // namespace specattn
