// What the two paths of specattn_kv4_verify share: the call's parameters, the partition of the work, the gather of
// rows into shared memory, and the ends of a unit.
#pragma once
#include <float.h>
#include <math.h>

#include "kv4.cuh"
#include "ptx.cuh"

namespace specattn {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kChunk = 32;  // positions that a warp gathers at a time
constexpr int kStageBytes = kChunk * (2 * kKv4Row + 8);
constexpr int kRowFloats = kKv4D + 4;  // a query row's record: output, maximum, sum, status (and 16-byte rows)
constexpr int kMaxUnits = 2048;
constexpr int kMaxPositions = 1 << 23;  // of a unit: chunks of all units are counted in 31 bits

struct Kv4Params {
  Kv4View cache;
  const unsigned char* q;
  const int *kv_len, *idx, *counts;
  long long idx_stride;
  unsigned char* out;
  float* lse;
  int* status;
  int* starts;     // workspace: first chunk of every unit, [units + 1], chunks of a CTA, the path taken
  int* flags;      // workspace: status of the units that one CTA has done, [units]; other units have it in their records
  float* partial;  // workspace: two records of a unit's rows for every CTA
  float scale;     // sm_scale * log2(e)
  int B, T, Hq, H, grp, rows, G, dense, tail, out_f32, half;
  int groups_of_rows, rows_per_group;  // of the mma.sync path
  int most_units;                      // of either path
  int engine, test_lose;               // 1: mma.sync, 2: tcgen05, 0: by the lengths
};

// The units of a path: (sequence, KV head), once for every group of query rows.
struct Units {
  int n, rows;  // units; query rows of one
};
__device__ __forceinline__ Units units_of(const Kv4Params& P, int tensor) {
  Units u;
  u.n = P.B * P.H * (tensor ? 1 : P.groups_of_rows);
  u.rows = tensor ? (P.rows + 7) / 8 * 8 : P.rows_per_group;
  return u;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 widen16(uint32_t pair, int half) { return half ? widen<true>(pair) : widen<false>(pair); }
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}

// Positions that sequence b, head h attends before the tail.
__device__ __forceinline__ int list_len(const Kv4Params& P, int b, int h) {
  if (P.dense) return max(0, min(P.kv_len[b], kMaxPositions));
  return static_cast<int>(max(0ll, min(static_cast<long long>(P.counts[b * P.G + (P.G > 1 ? h : 0)]), P.idx_stride)));
}
__device__ __forceinline__ int chunks_of(const Kv4Params& P, int u, int chunk) {
  const int bh = u % (P.B * P.H), b = bh / P.H;
  return (list_len(P, b, bh - b * P.H) + P.tail + chunk - 1) / chunk;
}

struct PartitionShared {
  int scan[33];
  int unit, unit_start, total;
};
// Chunks of `chunk` positions of all units in a row, cut into equal runs: this CTA's is [first, last), its first unit
// `unit` begins at chunk `start`.
struct Partition {
  int total, per, first, last, unit, start;
};
template <int kThreads>
__device__ __forceinline__ int count_chunks(const Kv4Params& P, int units, int chunk, PartitionShared& S, int* before) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per_thread = (units + kThreads - 1) / kThreads;
  const int u0 = min(tid * per_thread, units), u1 = min(u0 + per_thread, units);
  int sum = 0;
  for (int u = u0; u < u1; ++u) sum += chunks_of(P, u, chunk);
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) S.scan[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    const int x = lane < kThreads / 32 ? S.scan[lane] : 0;
    int y = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int z = __shfl_up_sync(0xffffffffu, y, o);
      if (lane >= o) y += z;
    }
    if (lane < kThreads / 32) S.scan[lane] = y - x;
    if (lane == 31) S.total = y;
    if (lane == 0) S.unit = units, S.unit_start = 0;
  }
  __syncthreads();
  *before = S.scan[warp] + incl - sum;
  return S.total;
}
template <int kThreads>
__device__ __forceinline__ Partition cut(const Kv4Params& P, int units, int chunk, int least, int tensor, PartitionShared& S, int total, int before) {
  Partition p;
  const int tid = threadIdx.x;
  p.total = total;
  p.per = max((total + static_cast<int>(gridDim.x) - 1) / static_cast<int>(gridDim.x), least);
  p.first = min(static_cast<long long>(blockIdx.x) * p.per, static_cast<long long>(total));
  p.last = min(p.first + p.per, total);
  const int per_thread = (units + kThreads - 1) / kThreads;
  const int u0 = min(tid * per_thread, units), u1 = min(u0 + per_thread, units);
  int run = before;
  for (int u = u0; u < u1; ++u) {
    const int n = chunks_of(P, u, chunk);
    if (blockIdx.x == 0) P.starts[u] = run;
    if (n > 0 && run <= p.first && p.first < run + n) S.unit = u, S.unit_start = run;
    run += n;
  }
  if (blockIdx.x == 0 && tid == 0) {
    P.starts[units] = total;
    P.starts[P.most_units + 1] = p.per;
    P.starts[P.most_units + 2] = tensor;
  }
  __syncthreads();
  p.unit = S.unit;
  p.start = S.unit_start;
  return p;
}

// The positions of one unit, looked up and fetched by warps.
struct Gather {
  const Kv4Params& P;
  int b, h, n_list, n_all, ctx;
  const int* list;

  __device__ __forceinline__ Gather(const Kv4Params& p, int b_, int h_) : P(p), b(b_), h(h_) {
    n_list = list_len(P, b, h);
    n_all = n_list + P.tail;
    ctx = max(0, P.kv_len[b]);
    list = P.dense ? nullptr : P.idx + (static_cast<long long>(b) * P.G + (P.G > 1 ? h : 0)) * P.idx_stride;
  }
  __device__ __forceinline__ int position(int i) const {  // the i-th position; -1: none, -2: out of range
    if (i >= n_all) return -1;
    if (i >= n_list) return ctx + (i - n_list);
    const int pos = P.dense ? i : list[i];
    return pos >= 0 && pos < ctx ? pos : -2;
  }
  __device__ __forceinline__ int page(int pos) const {
    if (pos == -1) return -1;
    if (pos >= 0) {
      const long long p = page_of(P.cache.table, P.cache.table_stride, P.cache.n_pages, b, pos / P.cache.by_page);
      if (p >= 0) return static_cast<int>(p);
    }
    return -2;
  }
  // A lane's position and page; the warp copies the 32 rows to a stage: K rows, V rows, then (s, z, t, y) of each.
  // `place_k` and `place_v`: where 16-byte piece t of row r goes, from the rows' beginning.
  template <typename PlaceK, typename PlaceV>
  __device__ __forceinline__ void fetch(uint32_t stage, int pos, int pg, int lane, int* bad, PlaceK place_k, PlaceV place_v) const {
    long long off = 0;
    int bytes = 0;
    const unsigned char* par = P.cache.params;
    if (pos != -1) {
      int slot = 0;
      if (pg < 0) {  // position 0 / page 0 in its place
        *bad = SPECATTN_ROW_BAD_INDEX;
        pg = 0;
      } else {
        slot = pos - pos / P.cache.by_page * P.cache.page_size;
      }
      off = pg * P.cache.s_page + slot * P.cache.s_slot + h * P.cache.s_head;
      par += pg * P.cache.p_page + slot * P.cache.p_slot + h * P.cache.p_head;
      bytes = 4;
    }
    // (a position that is none leaves zeros for scale and zero point, and any codes)
    cp_async4(stage + 2 * kChunk * kKv4Row + lane * 8, par, bytes);
    cp_async4(stage + 2 * kChunk * kKv4Row + lane * 8 + 4, par + P.cache.p_kv, bytes);
    const int t = lane & 3;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = j * 8 + (lane >> 2);
      const long long o = __shfl_sync(0xffffffffu, off, row);
      const unsigned char* from = P.cache.codes + o + t * 16;
      cp_async16(stage + place_k(row, t), from);
      cp_async16(stage + kChunk * kKv4Row + place_v(row, t), from + P.cache.s_kv);
    }
  }
};

// Query rows of a unit: byte offsets, what they see of the tail, their sums; and the power of two that takes the largest
// finite |q| to [2^14, 2^15): all 8 (or 11) bits of what lies within 2^-28 of it stay in fp16.
__device__ __forceinline__ long long query_at(const Kv4Params& P, int b, int h, int row) {
  const int tok = row / P.grp, hq = h * P.grp + row - tok * P.grp;
  return ((static_cast<long long>(b) * P.T + tok) * P.Hq + hq) * kKv4D;
}
template <int kWarps, int kQueries>
__device__ __forceinline__ void look_at_queries(const Kv4Params& P, int b, int h, int row0, int n_rows, int* qmax, float* qsum, int* limit) {
  const int lane = threadIdx.x & 31;
  for (int r = threadIdx.x >> 5; r < kQueries; r += kWarps) {
    float amax = 0.f, qs = 0.f;
    if (r < n_rows) {
      const uint2 x = *reinterpret_cast<const uint2*>(P.q + query_at(P, b, h, row0 + r) * 2 + lane * 8);
      const float2 a = widen16(x.x, P.half), c = widen16(x.y, P.half);
      qs = (a.x + a.y) + (c.x + c.y);
      const float v[4] = {fabsf(a.x), fabsf(a.y), fabsf(c.x), fabsf(c.y)};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v[e] <= FLT_MAX) amax = fmaxf(amax, v[e]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      qs += __shfl_xor_sync(0xffffffffu, qs, o);
    }
    if (lane == 0) {
      qsum[r] = r < n_rows ? qs * P.scale : 0.f;
      const int tok = r < n_rows ? (row0 + r) / P.grp : 0;
      limit[r] = max(0, min(P.tail, tok + P.tail - P.T + 1));
      atomicMax(qmax, __float_as_int(amax));
    }
  }
}
__device__ __forceinline__ int query_exponent(int qmax) {
  return min(14 - ((qmax >> 23) - 127), 120);  // (qmax is 0 or the bits of a positive number)
}
// Two 16-byte halves of eight neighbouring elements d ... d + 7 of a query row as fp16 operands against a word of codes:
// pairs (0, 4), (1, 5), (2, 6), (3, 7); what meets the high codes of a byte carries 2^-4.
__device__ __forceinline__ uint4 query_word(const Kv4Params& P, long long at, float up) {
  const uint4 x = *reinterpret_cast<const uint4*>(P.q + at * 2);
  const float2 a = widen16(x.x, P.half), b = widen16(x.y, P.half), c = widen16(x.z, P.half), d = widen16(x.w, P.half);
  const float hi = up * 0.0625f;
  return make_uint4(pack_f16(a.x * up, c.x * up), pack_f16(a.y * hi, c.y * hi), pack_f16(b.x * up, d.x * up), pack_f16(b.y * hi, d.y * hi));
}

// out and lse of a query row from its unnormalised output (four elements a lane), maximum and sum.
__device__ __forceinline__ void write_row(const Kv4Params& P, int b, int h, int row, int lane, const float4& o, float m, float l) {
  const long long at = query_at(P, b, h, row);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const float4 v = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  if (P.out_f32)
    *reinterpret_cast<float4*>(P.out + (at + 4 * lane) * 4) = v;
  else
    *reinterpret_cast<uint2*>(P.out + (at + 4 * lane) * 2) =
        P.half ? make_uint2(narrow<true>(v.x, v.y), narrow<true>(v.z, v.w)) : make_uint2(narrow<false>(v.x, v.y), narrow<false>(v.z, v.w));
  if (lane == 0) P.lse[at / kKv4D] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// The end of a segment: kParts records of every query row lie in `meet` ([part][kQueries][kRowFloats]); a warp joins a
// row's, a lane four elements, and writes the row, or its record if other CTAs work on the unit, too.
template <int kWarps, int kParts, int kQueries>
__device__ __forceinline__ void finish(const Kv4Params& P, const float* meet, int b, int h, int row0, int n_rows, bool whole, float* part) {
  const int lane = threadIdx.x & 31;
  for (int r = threadIdx.x >> 5; r < n_rows; r += kWarps) {
    float m = -FLT_MAX, l = 0.f;
#pragma unroll
    for (int w = 0; w < kParts; ++w) m = fmaxf(m, meet[(w * kQueries + r) * kRowFloats + kKv4D]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kParts; ++w) {
      const float* rec = meet + (w * kQueries + r) * kRowFloats;
      const float f = ex2(rec[kKv4D] - m);
      const float4 x = *reinterpret_cast<const float4*>(rec + 4 * lane);
      l = fmaf(f, rec[kKv4D + 1], l);
      o.x = fmaf(f, x.x, o.x), o.y = fmaf(f, x.y, o.y), o.z = fmaf(f, x.z, o.z), o.w = fmaf(f, x.w, o.w);
    }
    if (whole) {
      write_row(P, b, h, row0 + r, lane, o, m, l);
    } else {
      float* rec = part + r * kRowFloats;
      *reinterpret_cast<float4*>(rec + 4 * lane) = o;
      if (lane == 0) rec[kKv4D] = m, rec[kKv4D + 1] = l;
    }
  }
}

}  // namespace
}  // namespace specattn
