// specattn_kv4_verify: the attention of specattn_sparse_verify over a cache that holds its rows in 4 bits.
//
// The mathematics.  With K_i = s_i c_i + z_i and V_i = t_i e_i + y_i (codes c, e in 0..15),
//     q . K_i   = s_i (q . c_i) + z_i sum q
//     sum_i p_i V_i = sum_i (p_i t_i) (e_i - 8) + sum_i p_i (y_i + 8 t_i)
// so both products run over the codes themselves and the scales enter per (position, query) in binary32.  A code c
// as the bit pattern of an fp16 number is the subnormal c 2^-24, and 16 c is c 2^-20: masking a word of packed codes
// with 0x000f000f or 0x00f000f0 gives a register of two exact fp16 values and no conversion takes place (five
// instructions for eight codes; tensor cores take subnormals as they are).  Queries are scaled by a power of two so
// that they fit fp16 with all of their bits, those that meet the high codes of a byte by 2^-4 more.
// The second product is taken about the middle of the codes, by one more matrix instruction with a constant operand:
// the weights w = p t are rounded to fp16, and an error of w should be multiplied by a code's distance from 8, not
// by the code (2 to 3 times the error of the output).  And every second tile of positions uses 15 - e, the complement
// of the packed bits, with -w:  sum w e = sum_even w e + sum_odd (-w) (15 - e) + 15 sum_odd w.  The accumulators then
// stay near zero instead of growing with sum w, and what the matrix units cut off at each step stays as small (131072
// positions: the output's error falls from 1.6 times that of its rounding to bf16 to no more than it).
//
// The layout.  Positions are the rows of mma.m16n8k16 in the first product and the summed index in the second,
// queries the columns of both: 8 query rows cost one instruction where a form with queries as rows pays for 16.
// Which element of a row, and which of a tile's positions, goes to which lane is free as long as both operands
// agree, so a lane reads 16 bytes of a K row and 8 bytes of a V row as they lie in the cache.  Probabilities change
// from result to operand layout by movmatrix.
//
// A warp owns chunks of 32 positions from the gather to the running maximum, sum and output, with a ring of its own
// that cp.async fills: no barrier in the loop.  Warps meet at the end of a unit (sequence, KV head), CTAs through
// the workspace and a second kernel.
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "kv4.cuh"
#include "nvtx_range.h"
#include "ptx.cuh"

namespace specattn {

extern std::atomic<long long> g_launch_count;
int device_sm_count();

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kChunk = 32;        // positions of a chunk
constexpr int kStageBytes = kChunk * (2 * kKv4Row + 8);
constexpr int kRowFloats = kKv4D + 4;  // a query row's record in shared memory: output, maximum, sum (and 16-byte rows)
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
  int* starts;     // workspace: first chunk of every unit, [units + 1], then the chunks of a CTA
  int* flags;      // workspace: status of the units that one CTA has done, [units]; other units have it in their records
  float* partial;  // workspace: two records of a unit's rows for every CTA
  float scale;     // sm_scale * log2(e)
  int B, T, Hq, H, grp, rows, G, dense, tail, out_f32;
  int groups_of_rows, rows_per_group, units;
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
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

// Positions that unit (b, h) attends: its list, then the tail.
__device__ __forceinline__ int list_len(const Kv4Params& P, int b, int h) {
  if (P.dense) return max(0, min(P.kv_len[b], kMaxPositions));
  const int g = P.G > 1 ? h : 0;
  return static_cast<int>(max(0ll, min(static_cast<long long>(P.counts[b * P.G + g]), P.idx_stride)));
}

template <int NT, int NWARP, int STAGES, bool kHalf>
struct Kv4Kernel {
  static constexpr int kThreads = NWARP * 32;
  static constexpr int kQueries = NT * 8;
  static constexpr int kQBytes = NT * 8 * 32 * 8;  // query operand: [tile][step][lane] of two registers
  static constexpr int kRing = STAGES * kStageBytes;
  static constexpr int kMeet = NWARP * kQueries * kRowFloats * 4;  // what the warps leave for one another, in the rings' place
  static constexpr int kSmem = kQBytes + (NWARP * kRing > kMeet ? NWARP * kRing : kMeet);
};

template <int NT, int NWARP, int STAGES, bool kHalf>
__global__ void __launch_bounds__(NWARP * 32, 1) kv4_verify_kernel(const __grid_constant__ Kv4Params P) {
  using K = Kv4Kernel<NT, NWARP, STAGES, kHalf>;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int s_scan[NWARP + 1];
  __shared__ int s_unit, s_unit_start, s_total;
  __shared__ int s_bad[2];  // of this segment, and cleared for the next
  __shared__ int s_qmax;
  __shared__ float s_qsum[K::kQueries];
  __shared__ int s_limit[K::kQueries];  // how many tail positions a query row sees
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, t = lane & 3;
  unsigned char* ring = smem + K::kQBytes + warp * K::kRing;
  const uint32_t ring_at = smem_u32(ring);

  pdl_wait();  // everything below reads what earlier kernels may have written

  // ---- the partition: chunks of all units in a row, cut into equal runs ----
  const int per_thread = (P.units + K::kThreads - 1) / K::kThreads;
  const int u0 = min(tid * per_thread, P.units), u1 = min(u0 + per_thread, P.units);
  auto chunks_of = [&](int u) {
    const int bh = u % (P.B * P.H), b = bh / P.H;
    return (list_len(P, b, bh - b * P.H) + P.tail + kChunk - 1) / kChunk;
  };
  int sum = 0;
  for (int u = u0; u < u1; ++u) sum += chunks_of(u);
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) s_scan[warp] = incl;
  if (tid == 0) s_bad[0] = s_bad[1] = 0;
  __syncthreads();
  if (tid == 0) {
    int run = 0;
    for (int w = 0; w < NWARP; ++w) {
      const int x = s_scan[w];
      s_scan[w] = run;
      run += x;
    }
    s_total = run;
    s_unit = P.units;
  }
  __syncthreads();
  const int total = s_total;
  int per = (total + gridDim.x - 1) / gridDim.x;
  if (per < NWARP) per = NWARP;
  const int c0 = min(static_cast<int>(blockIdx.x) * per, total), c1 = min(c0 + per, total);
  {
    int run = s_scan[warp] + incl - sum;
    for (int u = u0; u < u1; ++u) {
      const int n = chunks_of(u);
      if (blockIdx.x == 0) P.starts[u] = run;
      if (n > 0 && run <= c0 && c0 < run + n) s_unit = u, s_unit_start = run;
      run += n;
    }
    if (blockIdx.x == 0 && tid == 0) P.starts[P.units] = total, P.starts[P.units + 1] = per;
  }
  __syncthreads();
  int u = s_unit, u_start = s_unit_start, turn = 0;

  // ---- one segment of a unit after the other ----
  for (int at = c0; at < c1;) {
    const int rg = u / (P.B * P.H), bh = u - rg * P.B * P.H, b = bh / P.H, h = bh - b * P.H;
    const int n_list = list_len(P, b, h), n_all = n_list + P.tail;
    const int n_chunks = (n_all + kChunk - 1) / kChunk;
    const int seg0 = at - u_start, seg1 = min(n_chunks, c1 - u_start);  // chunks of the unit
    const int ctx = max(0, P.kv_len[b]);
    const int* list = P.dense ? nullptr : P.idx + (static_cast<long long>(b) * P.G + (P.G > 1 ? h : 0)) * P.idx_stride;
    const int row0 = rg * P.rows_per_group, n_rows = min(P.rows_per_group, P.rows - row0);

    // gather: where a lane's position of a chunk lies
    auto position = [&](int chunk) -> int {  // -1: none, -2: out of range
      const int i = chunk * kChunk + lane;
      if (chunk >= seg1 || i >= n_all) return -1;
      if (i >= n_list) return ctx + (i - n_list);
      const int pos = P.dense ? i : list[i];
      return pos >= 0 && pos < ctx ? pos : -2;
    };
    auto page = [&](int pos) -> int {
      if (pos == -1) return -1;
      if (pos >= 0) {
        const long long p = page_of(P.cache.table, P.cache.table_stride, P.cache.n_pages, b, pos / P.cache.by_page);
        if (p >= 0) return static_cast<int>(p);
      }
      return -2;
    };
    auto fetch = [&](int chunk, int pos, int pg) {
      const uint32_t stage = ring_at + ((chunk / NWARP) % STAGES) * kStageBytes;
      long long off = 0;
      int bytes = 0;
      const unsigned char* par = P.cache.params;
      if (pos != -1) {
        int slot = 0;
        if (pg < 0) {  // position 0 / page 0 in its place
          s_bad[turn] = SPECATTN_ROW_BAD_INDEX;
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
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // four lanes a row.  K rows lie in order.  Row j of a V tile of 16 lies where the second product's lanes find
        // it without bank conflicts: 2 t -> t, 2 t + 1 -> t + 4 within eight, its 32-byte halves swapped by bit 1.
        const int row = j * 8 + g, r8 = row & 7, v_row = (row & ~7) | ((r8 >> 1) | ((r8 & 1) << 2));
        const long long o = __shfl_sync(0xffffffffu, off, row);
        const unsigned char* from = P.cache.codes + o + t * 16;
        cp_async16(stage + row * kKv4Row + t * 16, from);
        cp_async16(stage + (kChunk + v_row) * kKv4Row + ((t * 16) ^ ((v_row & 2) << 4)), from + P.cache.s_kv);
      }
    };

    // the first chunks are on their way before the queries are read
    const int first = seg0 + ((warp - seg0) % NWARP + NWARP) % NWARP;  // this warp's: chunk % NWARP == warp
    int pos_next, pg_next, pos_then;  // of chunk + (STAGES - 1) NWARP; of the one behind it
    {
      int pos[STAGES + 1], pg[STAGES];
#pragma unroll
      for (int s = 0; s <= STAGES; ++s) pos[s] = position(first + s * NWARP);
#pragma unroll
      for (int s = 0; s < STAGES; ++s) pg[s] = page(pos[s]);
#pragma unroll
      for (int s = 0; s < STAGES - 1; ++s) {
        if (first + s * NWARP < seg1) fetch(first + s * NWARP, pos[s], pg[s]);
        cp_commit();
      }
      pos_next = pos[STAGES - 1];
      pg_next = pg[STAGES - 1];
      pos_then = pos[STAGES];
    }

    // ---- queries: fp16 operands, sums, what a row sees of the tail ----
    if (tid == 0) s_qmax = 0;
    __syncthreads();
    if (tid == 0) s_bad[turn ^ 1] = 0;
    auto query = [&](int r) {  // byte offset of query row r of the group
      const int row = row0 + r, tok = row / P.grp, hq = h * P.grp + row - tok * P.grp;
      return ((static_cast<long long>(b) * P.T + tok) * P.Hq + hq) * (kKv4D * 2);
    };
    for (int r = warp; r < K::kQueries; r += NWARP) {
      float amax = 0.f, qs = 0.f;
      if (r < n_rows) {
        const uint2 x = *reinterpret_cast<const uint2*>(P.q + query(r) + lane * 8);
        const float2 a = widen<kHalf>(x.x), c = widen<kHalf>(x.y);
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
        s_qsum[r] = r < n_rows ? qs : 0.f;
        const int tok = r < n_rows ? (row0 + r) / P.grp : 0;
        s_limit[r] = max(0, min(P.tail, tok + P.tail - P.T + 1));
        atomicMax(&s_qmax, __float_as_int(amax));
      }
    }
    __syncthreads();
    // the largest finite |q| of the unit goes to [2^14, 2^15): all 8 (or 11) bits of what lies within 2^-28 of it stay
    int qexp = 0;
    {
      const int e = (s_qmax >> 23) - 127;  // (-127 for zeros and subnormals)
      qexp = min(14 - e, 120);
    }
    const float q_up = __int_as_float((127 + qexp) << 23);
    for (int i = tid; i < NT * 8 * 32; i += K::kThreads) {
      const int nt = i >> 8, ks = (i >> 5) & 7, l = i & 31, r = nt * 8 + (l >> 2);
      uint2 w = make_uint2(0u, 0u);
      if (r < n_rows) {
        // step 2 w meets codes 0, 4 (low halves of bytes) and 1, 5 (high) of word w of the lane's 16 bytes, step
        // 2 w + 1 codes 2, 6 and 3, 7
        const int d = (l & 3) * 32 + (ks >> 1) * 8 + (ks & 1) * 2;
        const uint32_t* q32 = reinterpret_cast<const uint32_t*>(P.q + query(r) + d * 2);
        const float2 a = widen<kHalf>(q32[0]), c = widen<kHalf>(q32[2]);  // d, d + 1; d + 4, d + 5
        w.x = pack_f16(a.x * q_up, c.x * q_up);
        w.y = pack_f16(a.y * q_up * 0.0625f, c.y * q_up * 0.0625f);
      }
      reinterpret_cast<uint2*>(smem)[i] = w;
    }
    __syncthreads();
    const float k_mul = P.scale * 16777216.f * __int_as_float((127 - qexp) << 23);  // codes are c 2^-24 in the product
    float sq[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      sq[nt][0] = s_qsum[nt * 8 + 2 * t] * P.scale;
      sq[nt][1] = s_qsum[nt * 8 + 2 * t + 1] * P.scale;
    }

    // ---- the chunks ----
    float acc[8][NT][4], acc8[NT][4];       // output by (element tile, query tile), less its middle
    float m[NT][2], l[NT][2], y[NT][2];     // running maximum (log2), sum of p, sum of p (y + 8 t)
    float up = 3e38f;                        // the weights' power of two: w = p t up
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc8[nt][e] = 0.f;
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) acc[mt][nt][e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) m[nt][e] = -FLT_MAX, l[nt][e] = 0.f, y[nt][e] = 0.f;
    }
    const uint2* q_op = reinterpret_cast<const uint2*>(smem) + lane;

#pragma unroll 1
    for (int chunk = first; chunk < seg1; chunk += NWARP) {
      cp_wait<STAGES - 2>();
      __syncwarp();
      {
        const int ahead = chunk + (STAGES - 1) * NWARP;
        if (ahead < seg1) fetch(ahead, pos_next, pg_next);
        cp_commit();
        pos_next = pos_then;
        pg_next = page(pos_then);
        pos_then = position(ahead + 2 * NWARP);
      }
      const uint32_t stage = ring_at + ((chunk / NWARP) % STAGES) * kStageBytes;

      // first product: scores of two tiles of 16 positions
      float s[2][NT][4];
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[h2][nt][e] = 0.f;
      {
        uint32_t ka[2][2][4];
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const uint4 x = lds128(stage + (h2 * 16 + r * 8 + g) * kKv4Row + t * 16);
            ka[h2][r][0] = x.x, ka[h2][r][1] = x.y, ka[h2][r][2] = x.z, ka[h2][r][3] = x.w;
          }
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int hi = 0; hi < 2; ++hi) {
            uint32_t a[2][4];
#pragma unroll
            for (int h2 = 0; h2 < 2; ++h2) {
              const uint32_t x0 = hi ? ka[h2][0][w] >> 8 : ka[h2][0][w], x1 = hi ? ka[h2][1][w] >> 8 : ka[h2][1][w];
              a[h2][0] = x0 & 0x000f000fu, a[h2][1] = x1 & 0x000f000fu;
              a[h2][2] = x0 & 0x00f000f0u, a[h2][3] = x1 & 0x00f000f0u;
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const uint2 qb = q_op[(nt * 8 + 2 * w + hi) * 32];
#pragma unroll
              for (int h2 = 0; h2 < 2; ++h2) mma_f16(s[h2][nt], a[h2][0], a[h2][1], a[h2][2], a[h2][3], qb.x, qb.y);
            }
          }
      }

      // scales: (s, z) and (t, y) of the positions g and g + 8 of both tiles
      float t_of[2][2], y_of[2][2], t_max = 0.f;
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint2 x = lds64(stage + 2 * kChunk * kKv4Row + (h2 * 16 + r * 8 + g) * 8);
          const float2 kp = widen<kHalf>(x.x), vp = widen<kHalf>(x.y);
          const float ks = kp.x * k_mul;
          t_of[h2][r] = vp.x;
          y_of[h2][r] = fmaf(8.f, vp.x, vp.y);
          t_max = fmaxf(t_max, fabsf(vp.x));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) s[h2][nt][2 * r + e] = fmaf(s[h2][nt][2 * r + e], ks, kp.y * sq[nt][e]);
        }
      // what a query does not see: past the end, or behind it in the tail
      const int i0 = chunk * kChunk;
      if (i0 + kChunk > n_list) {
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int i = i0 + h2 * 16 + r * 8 + g;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (i >= n_list + s_limit[nt * 8 + 2 * t + e]) s[h2][nt][2 * r + e] = -INFINITY;
          }
      }
      // the maximum moves only where a score passes it by 2^8, the weights' scale where one passes 64
      bool over = t_max * up > 64.f;
      float top[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          top[nt][e] = fmaxf(fmaxf(s[0][nt][e], s[0][nt][2 + e]), fmaxf(s[1][nt][e], s[1][nt][2 + e]));
          over = over || top[nt][e] > m[nt][e] + 8.f;
        }
      if (__any_sync(0xffffffffu, over)) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t_max = fmaxf(t_max, __shfl_xor_sync(0xffffffffu, t_max, o));
        // t_max up in [32, 64); finite t only
        const int e = (__float_as_int(t_max) >> 23) - 127;
        float up_now = up;
        if (t_max <= FLT_MAX && t_max > 0.f) up_now = fminf(up, __int_as_float((127 + min(5 - e, 100)) << 23));
        const float scale_now = up_now / up;
        up = up_now;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float f[2];
#pragma unroll
          for (int e2 = 0; e2 < 2; ++e2) {
            float v = top[nt][e2];
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
            const float m_now = fmaxf(m[nt][e2], v);
            f[e2] = ex2(m[nt][e2] - m_now);
            m[nt][e2] = m_now;
            l[nt][e2] *= f[e2];
            y[nt][e2] *= f[e2];
            f[e2] *= scale_now;
          }
#pragma unroll
          for (int e2 = 0; e2 < 4; ++e2) {
            acc8[nt][e2] *= f[e2 & 1];
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) acc[mt][nt][e2] *= f[e2 & 1];
          }
        }
      }

      // weights, and the second product
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2) {
        uint32_t pb[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float x = s[h2][nt][2 * r + e], p = ex2(x - m[nt][e]);
              // (a masked row may hold anything, NaN included)
              const bool none = x == -INFINITY;
              l[nt][e] += p;
              y[nt][e] = none ? y[nt][e] : fmaf(p, y_of[h2][r], y[nt][e]);
              w[e] = none ? 0.f : p * (t_of[h2][r] * up);
            }
            pb[nt][r] = transpose8(h2 ? pack_f16(-w[0], -w[1]) : pack_f16(w[0], w[1]));
          }
        // V rows of positions 2 t, 2 t + 1, 2 t + 8, 2 t + 9 of the tile, 8 bytes to a lane
        uint2 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int row = h2 * 16 + (k >> 1) * 8 + (k & 1) * 4 + t;
          v[k] = lds64(stage + (kChunk + row) * kKv4Row + ((g * 8) ^ ((row & 2) << 4)));
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint32_t mid = h2 ? 0x80078007u : 0x80088008u;  // -7 (of -w: 15 w - 8 w), -8
          mma_f16(acc8[nt], mid, mid, mid, mid, pb[nt][0], pb[nt][1]);
        }
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t sel = half ? 0x7632u : 0x5410u;
            uint32_t x0 = w ? __byte_perm(v[0].y, v[1].y, sel) : __byte_perm(v[0].x, v[1].x, sel);
            uint32_t x1 = w ? __byte_perm(v[2].y, v[3].y, sel) : __byte_perm(v[2].x, v[3].x, sel);
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
              const int mt = w * 4 + half * 2 + hi;
              if (hi) x0 >>= 8, x1 >>= 8;
              const uint32_t z0 = h2 ? ~x0 : x0, z1 = h2 ? ~x1 : x1;
              const uint32_t a0 = z0 & 0x000f000fu, a1 = z0 & 0x00f000f0u, a2 = z1 & 0x000f000fu, a3 = z1 & 0x00f000f0u;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma_f16(acc[mt][nt], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
            }
          }
      }
    }
    cp_wait<0>();
    __syncthreads();  // the rings are free

    // ---- the warps' parts meet: records of kRowFloats a query row ----
    float* meet = reinterpret_cast<float*>(smem + K::kQBytes);
    {
      const float down = 1.f / up;  // (0 where the warp has seen nothing: its sums are 0)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float ls = l[nt][e], ys = y[nt][e];
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) {
            ls += __shfl_xor_sync(0xffffffffu, ls, o);
            ys += __shfl_xor_sync(0xffffffffu, ys, o);
          }
          float* rec = meet + (warp * K::kQueries + nt * 8 + 2 * t + e) * kRowFloats;
          if (g == 0) rec[kKv4D] = m[nt][e], rec[kKv4D + 1] = ls;
          const float mid = acc8[nt][e];
          // lane g has elements 16 g ... 16 g + 15: tile mt holds 2 mt (codes in the low half of a byte) and 2 mt + 1
#pragma unroll
          for (int mt = 0; mt < 8; mt += 2) {
            float4 o4;
            o4.x = fmaf((acc[mt][nt][e] + mid) * 16777216.f, down, ys);
            o4.y = fmaf(fmaf(acc[mt][nt][2 + e], 1048576.f, mid * 16777216.f), down, ys);
            o4.z = fmaf((acc[mt + 1][nt][e] + mid) * 16777216.f, down, ys);
            o4.w = fmaf(fmaf(acc[mt + 1][nt][2 + e], 1048576.f, mid * 16777216.f), down, ys);
            *reinterpret_cast<float4*>(rec + 16 * g + 2 * mt) = o4;
          }
        }
    }
    __syncthreads();
    const bool whole = seg0 == 0 && seg1 == n_chunks;
    float* part = P.partial + static_cast<long long>(2 * blockIdx.x + (seg0 == 0 ? 1 : 0)) * K::kQueries * kRowFloats;
    // a warp has a row, a lane four elements
    for (int r = warp; r < n_rows; r += NWARP) {
      float M = -FLT_MAX;
#pragma unroll
      for (int w = 0; w < NWARP; ++w) M = fmaxf(M, meet[(w * K::kQueries + r) * kRowFloats + kKv4D]);
      float ls = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < NWARP; ++w) {
        const float* rec = meet + (w * K::kQueries + r) * kRowFloats;
        const float f = ex2(rec[kKv4D] - M);
        const float4 x = *reinterpret_cast<const float4*>(rec + 4 * lane);
        ls = fmaf(f, rec[kKv4D + 1], ls);
        o.x = fmaf(f, x.x, o.x), o.y = fmaf(f, x.y, o.y), o.z = fmaf(f, x.z, o.z), o.w = fmaf(f, x.w, o.w);
      }
      if (!whole) {
        float* rec = part + r * kRowFloats;
        *reinterpret_cast<float4*>(rec + 4 * lane) = o;
        if (lane == 0) rec[kKv4D] = M, rec[kKv4D + 1] = ls;
        continue;
      }
      const int row = row0 + r, tok = row / P.grp, hq = h * P.grp + row - tok * P.grp;
      const long long at_row = (static_cast<long long>(b) * P.T + tok) * P.Hq + hq;
      const float inv = ls == 0.f ? 0.f : 1.f / ls;
      if (P.out_f32)
        *reinterpret_cast<float4*>(P.out + (at_row * kKv4D + 4 * lane) * 4) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
      else
        *reinterpret_cast<uint2*>(P.out + (at_row * kKv4D + 4 * lane) * 2) =
            make_uint2(narrow<kHalf>(o.x * inv, o.y * inv), narrow<kHalf>(o.z * inv, o.w * inv));
      if (lane == 0) P.lse[at_row] = ls == 0.f ? -INFINITY : (M + log2f(ls)) * kLn2;
    }
    if (tid == 0) {
      if (whole)
        P.flags[u] = s_bad[turn];
      else
        part[kKv4D + 2] = __int_as_float(s_bad[turn]);
    }
    turn ^= 1;
    __syncthreads();  // the records have been read
    at = u_start + seg1;
    if (seg1 == n_chunks) {
      u_start += n_chunks;
      do {
        ++u;
      } while (u < P.units && at < c1 && chunks_of(u) == 0);
    }
  }
  pdl_launch_dependents();
}

// Joins the parts of units that several CTAs have worked on, and writes the rows of those that nobody has.
template <int NT, bool kHalf>
__global__ void __launch_bounds__(256) kv4_join_kernel(const __grid_constant__ Kv4Params P) {
  pdl_launch_dependents();
  pdl_wait();
  if (blockIdx.x == P.units) {  // the last block gathers the status words
    if (P.status == nullptr || blockIdx.y != 0) return;
    const int per_cta = P.starts[P.units + 1];
    for (int b = threadIdx.x >> 5; b < P.B; b += 8) {
      int flag = 0;
      for (int i = threadIdx.x & 31; i < P.H * P.groups_of_rows; i += 32) {
        const int unit = (i / P.H) * P.B * P.H + b * P.H + i % P.H, s0 = P.starts[unit], s1 = P.starts[unit + 1];
        if (s0 == s1) continue;
        const int f = s0 / per_cta, e = (s1 - 1) / per_cta;
        if (f == e) {
          flag |= P.flags[unit];
        } else {
          for (int c = f; c <= e; ++c)
            flag |= __float_as_int(P.partial[static_cast<long long>(2 * c + (c == f ? 1 : 0)) * (NT * 8 * kRowFloats) + kKv4D + 2]);
        }
      }
      flag = __reduce_or_sync(0xffffffffu, flag);
      if ((threadIdx.x & 31) == 0) P.status[b] = flag;
    }
    return;
  }
  const int u = blockIdx.x, lane = threadIdx.x & 31;
  const int c0 = P.starts[u], c1 = P.starts[u + 1], per = P.starts[P.units + 1];
  const int first = c0 / per, last = c1 > c0 ? (c1 - 1) / per : first;
  if (c1 > c0 && first == last) return;
  const int rg = u / (P.B * P.H), bh = u - rg * P.B * P.H, b = bh / P.H, h = bh - b * P.H;
  const int row0 = rg * P.rows_per_group, n_rows = min(P.rows_per_group, P.rows - row0);
  const int r = blockIdx.y * 8 + (threadIdx.x >> 5);
  if (r >= n_rows) return;
  constexpr int kRec = NT * 8 * kRowFloats;
  float M = -FLT_MAX, ls = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c1 > c0) {
    // (the part of the CTA where the unit begins is its second record, unless the CTA begins with the unit: that
    // is a second record, too; all others are first records)
    auto rec_of = [&](int c) { return P.partial + static_cast<long long>(2 * c + (c == first ? 1 : 0)) * kRec + r * kRowFloats; };
    for (int c = first + lane; c <= last; c += 32) M = fmaxf(M, rec_of(c)[kKv4D]);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, s));
#pragma unroll 4
    for (int c = first; c <= last; ++c) {
      const float* rec = rec_of(c);
      const float2 ml = *reinterpret_cast<const float2*>(rec + kKv4D);
      const float4 x = *reinterpret_cast<const float4*>(rec + 4 * lane);
      const float f = ex2(ml.x - M);
      ls = fmaf(f, ml.y, ls);
      o.x = fmaf(f, x.x, o.x), o.y = fmaf(f, x.y, o.y), o.z = fmaf(f, x.z, o.z), o.w = fmaf(f, x.w, o.w);
    }
  }
  const int row = row0 + r, tok = row / P.grp, hq = h * P.grp + row - tok * P.grp;
  const long long at_row = (static_cast<long long>(b) * P.T + tok) * P.Hq + hq;
  const float inv = ls == 0.f ? 0.f : 1.f / ls;
  if (P.out_f32)
    *reinterpret_cast<float4*>(P.out + (at_row * kKv4D + 4 * lane) * 4) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  else
    *reinterpret_cast<uint2*>(P.out + (at_row * kKv4D + 4 * lane) * 2) =
        make_uint2(narrow<kHalf>(o.x * inv, o.y * inv), narrow<kHalf>(o.z * inv, o.w * inv));
  if (lane == 0) P.lse[at_row] = ls == 0.f ? -INFINITY : (M + log2f(ls)) * kLn2;
}

struct Shape {
  int rows, groups, rows_per_group, nt;
};

Shape shape_of(const specattn_kv4_verify_args& A) {
  Shape s;
  s.rows = A.n_q * (A.n_q_heads / A.n_kv_heads);
  const int tiles = (s.rows + 7) / 8;
  s.groups = tiles > 4 ? 2 : 1;
  s.nt = (tiles + s.groups - 1) / s.groups;
  s.rows_per_group = s.nt * 8;
  return s;
}

int validate(const specattn_kv4_verify_args* args) {
  if (args == nullptr) return SPECATTN_ERR_NULL;
  if (args->struct_size != sizeof(specattn_kv4_verify_args)) return SPECATTN_ERR_STRUCT_SIZE;
  const specattn_kv4_verify_args& A = *args;
  if (A.batch < 0 || A.n_q < 1 || A.n_q_heads < 1 || A.n_kv_heads < 1 || A.n_groups < 1 || A.n_q_heads % A.n_kv_heads != 0 ||
      (A.n_groups != 1 && A.n_groups != A.n_kv_heads) || !(A.sm_scale >= 0.f) || A.tail_len < 0 || A.tail_len > 64 || A.reserved != 0)
    return SPECATTN_ERR_RANGE;
  const int cc = kv4_check(A.cache);
  if (cc != SPECATTN_OK) return cc;
  if (A.cache.n_pages > INT32_MAX) return SPECATTN_ERR_RANGE;
  if (A.head_dim != kKv4D || A.n_q > SPECATTN_MAX_QUERY_ROWS || A.n_q * (A.n_q_heads / A.n_kv_heads) > SPECATTN_MAX_QUERY_ROWS ||
      static_cast<long long>(A.batch) * A.n_kv_heads > kMaxUnits)
    return SPECATTN_ERR_UNSUPPORTED;
  return SPECATTN_OK;
}

// starts, the run's length and flags, then the records
size_t starts_bytes(const specattn_kv4_verify_args& A, const Shape& s) {
  return (static_cast<size_t>(A.batch) * A.n_kv_heads * s.groups * 2 + 2 + 63) / 64 * 256;
}
size_t workspace_bytes(const specattn_kv4_verify_args& A, const Shape& s, int sms) {
  return starts_bytes(A, s) + static_cast<size_t>(2) * sms * s.nt * 8 * kRowFloats * sizeof(float);
}

template <int NT, int NWARP, int STAGES, bool kHalf>
int launch(const Kv4Params& P, int sms, cudaStream_t stream) {
  using K = Kv4Kernel<NT, NWARP, STAGES, kHalf>;
  static std::atomic<unsigned long long> prepared{0};  // a bit per device
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return SPECATTN_ERR_CUDA;
  }
  if (!((prepared.load(std::memory_order_acquire) >> dev) & 1ull)) {
    if (cudaFuncSetAttribute(kv4_verify_kernel<NT, NWARP, STAGES, kHalf>, cudaFuncAttributeMaxDynamicSharedMemorySize, K::kSmem) != cudaSuccess) {
      cudaGetLastError();
      return SPECATTN_ERR_CUDA;
    }
    prepared.fetch_or(1ull << dev, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(sms);
  cfg.blockDim = dim3(K::kThreads);
  cfg.dynamicSmemBytes = K::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kv4_verify_kernel<NT, NWARP, STAGES, kHalf>, P) != cudaSuccess) {
    cudaGetLastError();
    return SPECATTN_ERR_CUDA;
  }
  cfg.gridDim = dim3(P.units + 1, NT);
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = 0;
  if (cudaLaunchKernelEx(&cfg, kv4_join_kernel<NT, kHalf>, P) != cudaSuccess) {
    cudaGetLastError();
    return SPECATTN_ERR_CUDA;
  }
  g_launch_count.fetch_add(2, std::memory_order_relaxed);
  return SPECATTN_OK;
}

template <bool kHalf>
int launch_of(const Kv4Params& P, int nt, int sms, cudaStream_t stream) {
  switch (nt) {
    case 1: return launch<1, 8, 4, kHalf>(P, sms, stream);
    case 2: return launch<2, 8, 4, kHalf>(P, sms, stream);
    case 3: return launch<3, 8, 4, kHalf>(P, sms, stream);
    default: return launch<4, 8, 4, kHalf>(P, sms, stream);
  }
}

}  // namespace
}  // namespace specattn

extern "C" size_t specattn_kv4_verify_workspace_bytes(const specattn_kv4_verify_args* args) {
  if (specattn::validate(args) != SPECATTN_OK) return 0;
  const int sms = specattn::device_sm_count();
  if (sms <= 0) return 0;
  return specattn::workspace_bytes(*args, specattn::shape_of(*args), sms);
}

extern "C" int specattn_kv4_verify(const specattn_kv4_verify_args* args, void* cuda_stream) {
  using namespace specattn;
  NvtxRange nvtx_range("specattn_kv4_verify");
  const int v = validate(args);
  if (v != SPECATTN_OK) return v;
  const specattn_kv4_verify_args& A = *args;
  if (A.batch == 0) return SPECATTN_OK;
  if (!A.q || !A.kv_len || !A.out || !A.lse || !A.workspace) return SPECATTN_ERR_NULL;
  if (!A.dense && (!A.idx || !A.counts)) return SPECATTN_ERR_NULL;
  if (!A.dense && A.idx_stride < 0) return SPECATTN_ERR_RANGE;
  if ((!A.dense && A.idx_stride > kMaxPositions) ||
      (A.dense && A.cache.block_table_stride > kMaxPositions / A.cache.page_size))
    return SPECATTN_ERR_UNSUPPORTED;
  const int cb = kv4_check_buffers(A.cache);
  if (cb != SPECATTN_OK) return cb;
  if (reinterpret_cast<uintptr_t>(A.q) % 16 != 0 || reinterpret_cast<uintptr_t>(A.out) % 16 != 0 ||
      reinterpret_cast<uintptr_t>(A.workspace) % 256 != 0)
    return SPECATTN_ERR_ALIGN;
  const int sms = device_sm_count();
  if (sms <= 0) return SPECATTN_ERR_CUDA;
  const Shape s = shape_of(A);
  if (A.workspace_bytes < workspace_bytes(A, s, sms)) return SPECATTN_ERR_WORKSPACE;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  Kv4Params P;
  memset(&P, 0, sizeof(P));
  P.cache = kv4_view(A.cache);
  P.q = static_cast<const unsigned char*>(A.q);
  P.kv_len = A.kv_len;
  P.idx = A.idx;
  P.counts = A.counts;
  P.idx_stride = A.idx_stride;
  P.out = static_cast<unsigned char*>(A.out);
  P.lse = A.lse;
  P.status = A.status;
  P.units = A.batch * A.n_kv_heads * s.groups;
  P.starts = static_cast<int*>(A.workspace);
  P.flags = P.starts + P.units + 2;
  P.partial = reinterpret_cast<float*>(static_cast<unsigned char*>(A.workspace) + starts_bytes(A, s));
  P.scale = (A.sm_scale != 0.f ? A.sm_scale : 1.0f / sqrtf(static_cast<float>(A.head_dim))) * kLog2e;
  P.B = A.batch;
  P.T = A.n_q;
  P.Hq = A.n_q_heads;
  P.H = A.n_kv_heads;
  P.grp = A.n_q_heads / A.n_kv_heads;
  P.rows = s.rows;
  P.G = A.n_groups;
  P.dense = A.dense ? 1 : 0;
  P.tail = A.tail_len;
  P.out_f32 = A.out_f32 ? 1 : 0;
  P.groups_of_rows = s.groups;
  P.rows_per_group = s.rows_per_group;
  return A.cache.dtype == SPECATTN_DTYPE_FP16 ? launch_of<true>(P, s.nt, sms, stream) : launch_of<false>(P, s.nt, sms, stream);
}
