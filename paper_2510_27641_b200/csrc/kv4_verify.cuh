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
  int2* parts;     // workspace: first and last CTA of every unit, (0, -1) where it has no positions
  int* flags;      // workspace: status of the units that one CTA has done, [units]; other units have it in their records
  float* partial;  // workspace: two records of a unit's rows for every CTA
  float scale;     // sm_scale * log2(e)
  int B, T, Hq, H, grp, rows, G, dense, tail, out_f32, half;
  int n_units, rows_per_unit;
  unsigned c_page, c_slot, p_page, p_slot;  // strides of codes in 16-byte, of params in 4-byte units
  int pages_per_seq;
  int test_lose;
};

// A value that all lanes share, in a register that the warp shares.
__device__ __forceinline__ int uniform(int x) { return static_cast<int>(__reduce_or_sync(0xffffffffu, static_cast<unsigned>(x))); }

// The units of a path: (sequence, KV head), once for every group of query rows.
struct Units {
  int n, rows;  // units; query rows of one
};
__device__ __forceinline__ Units units_of(const Kv4Params& P) { return {P.n_units, P.rows_per_unit}; }

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Two numbers as sums of two fp16 numbers each, off by 2^-21 of themselves or 2^-24, whichever is more: their first 11 bits, and
// the rest, rounded.  (Cut, not rounded: a mask takes the place of a conversion back; 8 x 32768, 40 rows on tcgen05
// 179 against 171 us, 24 on mma.sync 142 against 138.)
__device__ __forceinline__ uint2 halves_f16(float lo, float hi) {
  const float lo11 = __uint_as_float(__float_as_uint(lo) & 0xffffe000u), hi11 = __uint_as_float(__float_as_uint(hi) & 0xffffe000u);
  return make_uint2(pack_f16(lo11, hi11), pack_f16(lo - lo11, hi - hi11));
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
  if (P.dense) return max(0, min(P.kv_len[b], kMaxPositions + 1));  // (the last of these is beyond any table)
  return static_cast<int>(max(0ll, min(static_cast<long long>(P.counts[b * P.G + (P.G > 1 ? h : 0)]), P.idx_stride)));
}
__device__ __forceinline__ int chunks_of(const Kv4Params& P, int u, int chunk) {
  const int bh = u % (P.B * P.H), b = bh / P.H;
  return (list_len(P, b, bh - b * P.H) + P.tail + chunk - 1) / chunk;
}

constexpr int kMostParted = 256;  // units that may be cut into equal parts
struct PartitionShared {
  int scan[33];
  int unit, unit_start, first, last;
  int chunks[kMostParted], parts[16];
};
// The units' chunks of `chunk` positions in a row, cut.  This CTA's run is [first, last), the chunks of its first unit, `unit`,
// begin at `start`, and `between` places lie in front of every unit's chunks.
struct Partition {
  int first, last, unit, start, between;
};

// The exclusive prefix of v over the threads of the CTA; the total in *total.
template <int kThreads>
__device__ __forceinline__ int scan(int v, PartitionShared& S, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();  // the last scan's sums have been read
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
    if (lane == 31) S.scan[32] = y;
  }
  __syncthreads();
  *total = S.scan[32];
  return S.scan[warp] + incl - v;
}

// Two ways to cut.  Equal runs of all units one after the other, each with `afresh` places in front of its chunks, as many chunks
// as the end of one unit and the start of the next take: a CTA that meets many short units has fewer chunks (20 rows over 32
// ragged lists of 631 to 16000: 146 to 91 us).  Or, where there are CTAs enough, equal parts of units: of lengths from an equal
// share of the chunks on, in steps of an eighth, each tried by a warp, the shortest whose parts are no more than the CTAs, if it exceeds
// that share by less than `afresh`.
template <int kThreads>
__device__ __forceinline__ Partition cut(const Kv4Params& P, int chunk, int least, int afresh, PartitionShared& S) {
  static_assert(kThreads >= kMostParted && kThreads <= 512, "a unit to a thread, a length to a warp");
  const int tid = threadIdx.x, lane = tid & 31, grid = static_cast<int>(gridDim.x), units = units_of(P).n;
  const int per_thread = (units + kThreads - 1) / kThreads;
  const int u0 = min(tid * per_thread, units), u1 = min(u0 + per_thread, units);
  int mine = 0, last_n = 0, total;
  for (int u = u0; u < u1; ++u) {
    last_n = chunks_of(P, u, chunk);
    mine += last_n > 0 ? last_n + afresh : 0;
  }
  if (tid < kMostParted) S.chunks[tid] = last_n;  // (read where a thread has one unit)
  if (tid == 0) S.unit = units;
  const int before = scan<kThreads>(mine, S, &total);
  Partition p;
  p.unit = units;
  p.start = p.first = p.last = 0;
  p.between = afresh;
  if (units <= min(grid, kMostParted)) {
    const int chunks = total - afresh * __syncthreads_count(last_n > 0);
    const int share = max((chunks + grid - 1) / grid, least);
    const auto length_of = [&](int step) { return share + share * step / 8; };
    {
      const int warp = tid >> 5;
      int n = 0;
      for (int u = lane; u < units; u += 32) n += (S.chunks[u] + length_of(warp) - 1) / length_of(warp);
      n = __reduce_add_sync(0xffffffffu, n);
      if (lane == 0) S.parts[warp] = n;
    }
    __syncthreads();
    int step = 0;
    while (step < kThreads / 32 && S.parts[step] > grid) ++step;
    if (step < kThreads / 32 && length_of(step) - share < afresh) {
      const int k = (last_n + length_of(step) - 1) / length_of(step);
      int all;
      const int at = scan<kThreads>(k, S, &all);  // this thread's unit goes to CTAs at ... at + k - 1
      if (tid < units) {
        if (blockIdx.x == 0) P.parts[tid] = k > 0 ? make_int2(at, at + k - 1) : make_int2(0, -1);
        const int j = static_cast<int>(blockIdx.x) - at;
        if (j >= 0 && j < k) {
          S.unit = tid;
          S.first = static_cast<int>(static_cast<long long>(last_n) * j / k);
          S.last = static_cast<int>(static_cast<long long>(last_n) * (j + 1) / k);
        }
      }
      __syncthreads();
      if (S.unit < units) p.unit = S.unit, p.first = S.first, p.last = S.last;
      return p;
    }
  }
  const int per = max((total + grid - 1) / grid, least);
  const int from = static_cast<int>(min(static_cast<long long>(blockIdx.x) * per, static_cast<long long>(total)));
  p.last = min(from + per, total);
  int run = before;
  for (int u = u0; u < u1; ++u) {
    const int n = chunks_of(P, u, chunk);
    if (n > 0) run += afresh;  // where the unit's chunks begin
    if (blockIdx.x == 0) P.parts[u] = n > 0 ? make_int2(run / per, (run + n - 1) / per) : make_int2(0, -1);
    if (n > 0 && run - afresh <= from && from < run + n) S.unit = u, S.unit_start = run;
    run += n;
  }
  __syncthreads();
  p.unit = S.unit;
  p.start = S.unit_start;
  p.first = max(from, p.start);
  return p;
}

// The positions of one unit, looked up and fetched by warps.  Rows are addressed in 16-byte (codes) and 4-byte
// (params) units of 32 bits, which reach 64 GB of codes: a lookup is a dozen instructions instead of fifty.
struct Gather {
  const Kv4Params& P;
  int n_list, n_all, ctx;
  const int *list, *table;
  const unsigned char *codes, *params;  // of this head
  int first_page;                       // without a table

  __device__ __forceinline__ Gather(const Kv4Params& p, int b, int h) : P(p) {
    n_list = uniform(list_len(P, b, h));
    n_all = n_list + P.tail;
    ctx = uniform(max(0, P.kv_len[b]));
    list = P.dense ? nullptr : P.idx + (static_cast<long long>(b) * P.G + (P.G > 1 ? h : 0)) * P.idx_stride;
    table = P.cache.table != nullptr ? P.cache.table + b * P.cache.table_stride : nullptr;
    first_page = static_cast<int>(min(b * P.cache.table_stride, P.cache.n_pages));  // (n_pages fits; beyond it no page is)
    codes = P.cache.codes + h * P.cache.s_head;
    params = P.cache.params + h * P.cache.p_head;
  }
  // The three steps to the i-th row, made a tile or more apart: what a step loads is looked at by the next one only, since a
  // warp that compared it at once would wait for it (900 cycles a tile).
  __device__ __forceinline__ int position(int i) const {
    if (i >= n_all) return 0;
    return i >= n_list ? ctx + (i - n_list) : P.dense ? i : list[i];
  }
  __device__ __forceinline__ int page(int i, int pos) const {  // -2: none
    const int pi = pos / P.cache.by_page;  // (of a negative position: anything)
    if (i >= n_all || pos < 0 || (i < n_list && pos >= ctx) || pi >= P.pages_per_seq) return -2;
    return table != nullptr ? table[pi] : static_cast<int>(static_cast<unsigned>(first_page) + pi);
  }
  // Where the row lies: units from `codes` and `params`.  Position 0 / page 0 where position or page is out of range.
  __device__ __forceinline__ uint2 locate(int i, int pos, int pg, int* bad) const {
    if (i >= n_all) return make_uint2(0u, 0u);
    unsigned slot = static_cast<unsigned>(pos - pos / P.cache.by_page * P.cache.page_size);
    if (static_cast<unsigned>(pg) >= static_cast<unsigned>(P.cache.n_pages)) {
      *bad = SPECATTN_ROW_BAD_INDEX;
      pg = 0;
      slot = 0;
    }
    return make_uint2(pg * P.c_page + slot * P.c_slot, pg * P.p_page + slot * P.p_slot);
  }
  __device__ __forceinline__ const unsigned char* code_row(uint32_t at) const { return codes + static_cast<unsigned long long>(at) * 16; }
  __device__ __forceinline__ const unsigned char* param_row(uint32_t at) const { return params + static_cast<unsigned long long>(at) * 4; }
};

// A query row's first element.
__device__ __forceinline__ long long query_at(const Kv4Params& P, int b, int h, int row) {
  const int tok = row / P.grp, hq = h * P.grp + row - tok * P.grp;
  return ((static_cast<long long>(b) * P.T + tok) * P.Hq + hq) * kKv4D;
}

// The query rows of a unit as fp16 operands: a warp has every kWarps-th row, a lane four elements of it.  load() asks for
// them; look() finds sums, what the rows see of the tail, and the largest finite |q|; and, behind a barrier, place() writes
// them, scaled by the power of two that takes that largest to [2^14, 2^15): all 8 (or 11) bits of what lies within 2^-28
// of it stay.  Against a word of codes go pairs of elements (0, 4), (1, 5) from an even lane and (2, 6), (3, 7) from
// an odd one; the second of each meets the high codes of a byte and carries 2^-4.
template <int kWarps, int kQueries>
struct Queries {
  static constexpr int kMine = (kQueries + kWarps - 1) / kWarps;
  uint2 x[kMine];

  __device__ __forceinline__ void load(const Kv4Params& P, int b, int h, int row0, int n_rows) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int r = warp + i * kWarps;
      x[i] = r < n_rows ? *reinterpret_cast<const uint2*>(P.q + query_at(P, b, h, row0 + r) * 2 + lane * 8) : make_uint2(0u, 0u);
    }
  }
  __device__ __forceinline__ void look(const Kv4Params& P, int row0, int n_rows, int* qmax, float* qsum, int* limit) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int r = warp + i * kWarps;
      const float2 a = widen16(x[i].x, P.half), c = widen16(x[i].y, P.half);
      float qs = (a.x + a.y) + (c.x + c.y);
      const float v[4] = {fabsf(a.x), fabsf(a.y), fabsf(c.x), fabsf(c.y)};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v[e] <= FLT_MAX) most = fmaxf(most, v[e]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) qs += __shfl_xor_sync(0xffffffffu, qs, o);
      if (lane == 0 && r < kQueries) {
        qsum[r] = qs * P.scale;
        const int tok = r < n_rows ? (row0 + r) / P.grp : 0;
        limit[r] = max(0, min(P.tail, tok + P.tail - P.T + 1));
      }
    }
    const int top = __reduce_max_sync(0xffffffffu, __float_as_int(most));  // (bits of a number that is not negative)
    if (lane == 0) atomicMax(qmax, top);
  }
  // to(row, word, half, operand): word 0..15 of eight elements, its half of two registers
  template <typename To>
  __device__ __forceinline__ void place(const Kv4Params& P, float up, To to) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float hi = up * 0.0625f;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int r = warp + i * kWarps;
      const bool odd = lane & 1;
      const uint32_t other = __shfl_xor_sync(0xffffffffu, odd ? x[i].x : x[i].y, 1);
      const float2 a = widen16(odd ? other : x[i].x, P.half), c = widen16(odd ? x[i].y : other, P.half);
      if (r < kQueries) to(r, lane >> 1, lane & 1, make_uint2(pack_f16(a.x * up, c.x * up), pack_f16(a.y * hi, c.y * hi)));
    }
  }
};
__device__ __forceinline__ int query_exponent(int qmax) {
  return min(14 - ((qmax >> 23) - 127), 120);  // (qmax is 0 or the bits of a positive number)
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
