// The path of specattn_kv4_verify on mma.sync.
//
// The layout.  Positions are the rows of mma.m16n8k16 in the first product and the summed index in the second,
// queries the columns of both: 8 query rows cost one instruction where a form with queries as rows pays for 16.
// Which element of a row, and which of a tile's positions, goes to which lane is free as long as both operands
// agree, so a lane reads 16 bytes of a K row and 8 bytes of a V row as they lie in the cache.  Probabilities change
// from result to operand layout by movmatrix.
//
// The second eight positions of a tile use 15 - e, the complement of the packed bits, with -w:
//     sum_i p_i V_i = sum_first w e + sum_second (-w) (15 - e) + sum_first p y + sum_second p (y + 15 t).
// What an instruction adds is then around zero, and so are the accumulators, instead of growing with sum w: the matrix units cut
// off towards zero as they add, and a sum of one sign loses a little every time.
//
// A warp owns chunks of 32 positions from the gather to the running maximum, sum and output, with a ring of its own
// that cp.async fills: no barrier in the loop.  Warps meet at the end of a unit (sequence, KV head).
#pragma once
#include "kv4_verify.cuh"

namespace specattn {
namespace {

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

template <int NT, int NWARP, int STAGES>
struct MmaPath {
  static constexpr int kQueries = NT * 8;
  static constexpr int kQBytes = NT * 8 * 32 * 8;  // query operand: [tile][step][lane] of two registers
  static constexpr int kRing = STAGES * kStageBytes;
  static constexpr int kMeet = NWARP * kQueries * kRowFloats * 4;  // what the warps leave for one another, in the rings' place
  static constexpr int kSmem = kQBytes + (NWARP * kRing > kMeet ? NWARP * kRing : kMeet);
};

template <int kQueries>
struct MmaShared {
  int bad[2], qmax[2];  // of this segment, and cleared for the next
  float qsum[kQueries];  // times the scale
  int limit[kQueries];   // how many tail positions a query row sees
};

// kSpare: a call of up to four query rows, whose weights' remainders take the columns of the four that there are not (those of
// query q column 4 + q), and no instructions of their own.
template <int NT, int NWARP, int STAGES, bool kSpare>
__device__ __forceinline__ void mma_path(const Kv4Params& P, const Partition& part, unsigned char* smem, MmaShared<NT * 8>& S) {
  using K = MmaPath<NT, NWARP, STAGES>;
  const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
  const int g = lane >> 2, t = lane & 3;
  static_assert(!kSpare || NT == 1, "four columns to spare");
  const bool rests = kSpare && t >= 2;  // whose columns of the output are sums of remainders
  const uint32_t ring_at = smem_u32(smem + K::kQBytes + warp * K::kRing);
  const Units units = units_of(P);
  const int last = uniform(part.last);
  int u = uniform(part.unit), u_start = uniform(part.start), turn = 0;

  // ---- one segment of a unit after the other ----
  for (int at = uniform(part.first); at < last;) {
    const int rg = u / (P.B * P.H), bh = u - rg * P.B * P.H, b = bh / P.H, h = bh - b * P.H;
    const Gather G(P, b, h);
    const int n_list = G.n_list, n_chunks = (G.n_all + kChunk - 1) / kChunk;
    const int seg0 = at - u_start, seg1 = min(n_chunks, last - u_start);  // chunks of the unit
    const int row0 = rg * units.rows, n_rows = min(units.rows, P.rows - row0);

    auto position = [&](int chunk) { return chunk < seg1 ? G.position(chunk * kChunk + lane) : 0; };
    auto page = [&](int chunk, int pos) { return chunk < seg1 ? G.page(chunk * kChunk + lane, pos) : -2; };
    // The warp copies its 32 rows to a stage: K rows, V rows, then (s, z, t, y) of each.
    auto fetch = [&](int chunk, int pos, int pg) {
      const uint32_t stage = ring_at + ((chunk / NWARP) % STAGES) * kStageBytes;
      const uint2 row_at = G.locate(chunk * kChunk + lane, pos, pg, &S.bad[turn]);
      const unsigned char* par = G.param_row(row_at.y);
      const int bytes = chunk * kChunk + lane < G.n_all ? 4 : 0;  // (a position that is none leaves zeros for scale and zero point, and any codes)
      cp_async4(stage + 2 * kChunk * kKv4Row + lane * 8, par, bytes);
      cp_async4(stage + 2 * kChunk * kKv4Row + lane * 8 + 4, par + P.cache.p_kv, bytes);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // four lanes a row.  K rows lie in order.  Row j of a V tile of 16 lies where the second product's lanes find
        // it without bank conflicts: 2 t -> t, 2 t + 1 -> t + 4 within eight, its 32-byte halves swapped by bit 1.
        const int row = j * 8 + g, r8 = row & 7, v_row = (row & ~7) | ((r8 >> 1) | ((r8 & 1) << 2));
        const unsigned char* from = G.code_row(__shfl_sync(0xffffffffu, row_at.x, row) + t);
        cp_async16(stage + row * kKv4Row + t * 16, from);
        cp_async16(stage + (kChunk + v_row) * kKv4Row + ((t * 16) ^ ((v_row & 2) << 4)), from + P.cache.s_kv);
      }
    };

    Queries<NWARP, K::kQueries> queries;
    queries.load(P, b, h, row0, n_rows);
    // the first chunks are on their way before the queries are read
    const int first = seg0 + ((warp - seg0) % NWARP + NWARP) % NWARP;  // this warp's: chunk % NWARP == warp
    int pos_next, pg_next, pos_then;  // of chunk + (STAGES - 1) NWARP; of the one behind it
    {
      int pos[STAGES + 1], pg[STAGES];
#pragma unroll
      for (int s = 0; s <= STAGES; ++s) pos[s] = position(first + s * NWARP);
#pragma unroll
      for (int s = 0; s < STAGES; ++s) pg[s] = page(first + s * NWARP, pos[s]);
#pragma unroll
      for (int s = 0; s < STAGES - 1; ++s) {
        if (first + s * NWARP < seg1) fetch(first + s * NWARP, pos[s], pg[s]);
        cp_commit();
      }
      pos_next = pos[STAGES - 1];
      pg_next = pg[STAGES - 1];
      pos_then = pos[STAGES];
    }

    // ---- queries ----
    queries.look(P, row0, n_rows, &S.qmax[turn], S.qsum, S.limit);
    __syncthreads();
    if (tid == 0) S.bad[turn ^ 1] = S.qmax[turn ^ 1] = 0;
    const int qexp = query_exponent(S.qmax[turn]);
    // step 2 w meets codes 0, 4 (low halves of bytes) and 1, 5 (high) of word w of the lane's 16 bytes, step 2 w + 1
    // codes 2, 6 and 3, 7
    queries.place(P, __int_as_float((127 + qexp) << 23), [&](int r, int word, int half, uint2 x) {
      reinterpret_cast<uint2*>(smem)[((r >> 3) * 8 + 2 * (word & 3) + half) * 32 + (r & 7) * 4 + (word >> 2)] = x;
    });
    __syncthreads();
    const float k_mul = P.scale * 16777216.f * __int_as_float((127 - qexp) << 23);  // codes are c 2^-24 in the product
    Two sq[NT], m[NT], l[NT], y[NT];  // of two queries: sum q; minus the running maximum (log2), sum of p, sum of p (y + 0 or 15 t)
    float acc[8][NT][4];                             // output by (element tile, query tile), less what y has
    float up = 3e38f;                                // the weights' power of two: w = p t up
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) acc[mt][nt][e] = 0.f;
      }
      sq[nt] = two(S.qsum[nt * 8 + 2 * t], S.qsum[nt * 8 + 2 * t + 1]);
      m[nt] = l[nt] = y[nt] = two(0.f, 0.f);
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
        pg_next = page(ahead + NWARP, pos_then);
        pos_then = position(ahead + 2 * NWARP);
      }
      const uint32_t stage = ring_at + ((chunk / NWARP) % STAGES) * kStageBytes;

      // two tiles of 16 positions, one after the other: a loop of both would not fit the instruction caches
#pragma unroll 1
      for (int h2 = 0; h2 < 2; ++h2) {
        // first product
        const uint32_t k_row = stage + (h2 * 16 + g) * kKv4Row + t * 16;
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
        {
          const uint4 k0 = lds128(k_row), k1 = lds128(k_row + 8 * kKv4Row);
          const uint32_t ka[2][4] = {{k0.x, k0.y, k0.z, k0.w}, {k1.x, k1.y, k1.z, k1.w}};
#pragma unroll
          for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
              const uint32_t x0 = hi ? ka[0][w] >> 8 : ka[0][w], x1 = hi ? ka[1][w] >> 8 : ka[1][w];
              const uint32_t a0 = x0 & 0x000f000fu, a1 = x1 & 0x000f000fu, a2 = x0 & 0x00f000f0u, a3 = x1 & 0x00f000f0u;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                const uint2 qb = q_op[(nt * 8 + 2 * w + hi) * 32];
                mma_f16(s[nt], a0, a1, a2, a3, qb.x, qb.y);
              }
            }
        }

        // scales: (s, z) and (t, y) of the positions g and g + 8; scores from the running maximum on
        float t_of[2], y_of[2];
        {
          const uint32_t at_par = stage + 2 * kChunk * kKv4Row + (h2 * 16 + g) * 8;
          const uint2 raw[2] = {lds64(at_par), lds64(at_par + 64)};
          float2 kp[2], vp[2];
          if (P.half) {
#pragma unroll
            for (int r = 0; r < 2; ++r) kp[r] = widen<true>(raw[r].x), vp[r] = widen<true>(raw[r].y);
          } else {
#pragma unroll
            for (int r = 0; r < 2; ++r) kp[r] = widen<false>(raw[r].x), vp[r] = widen<false>(raw[r].y);
          }
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float ks = kp[r].x * k_mul;
            t_of[r] = vp[r].x;
            y_of[r] = r ? fmaf(15.f, vp[r].x, vp[r].y) : vp[r].y;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const float2 x2 = each(fma2(two(s[nt][2 * r], s[nt][2 * r + 1]), two(ks, ks), fma2(two(kp[r].y, kp[r].y), sq[nt], m[nt])));
              s[nt][2 * r] = x2.x, s[nt][2 * r + 1] = x2.y;
            }
          }
        }
        // what a query does not see: past the end, or behind it in the tail.  (A masked row may hold anything, and 0 NaN is
        // NaN: what a tail row's V scale would spoil, its scores spoil instead.)
        const int i0 = chunk * kChunk + h2 * 16;
        if (__builtin_expect(i0 + 16 > n_list, 0)) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int i = i0 + r * 8 + g;
            const bool spoilt = i >= n_list && !(fabsf(t_of[r]) <= FLT_MAX && fabsf(y_of[r]) <= FLT_MAX);
            if (spoilt) t_of[r] = y_of[r] = 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                if (spoilt) s[nt][2 * r + e] = NAN;
                if (i >= n_list + S.limit[nt * 8 + 2 * t + e]) s[nt][2 * r + e] = -INFINITY;
              }
          }
        }
        // the maximum moves only where a score passes it by 2^8, the weights' scale where one passes 64
        float top = s[0][0], t_max = fmaxf(fabsf(t_of[0]), fabsf(t_of[1]));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = fmaxf(top, s[nt][e]);
        const bool begins = chunk == first && h2 == 0;
        if (__builtin_expect(__any_sync(0xffffffffu, top > 8.f || t_max * up > 64.f || begins), 0)) {
          t_max = t_max <= FLT_MAX ? t_max : 0.f;
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) t_max = fmaxf(t_max, __shfl_xor_sync(0xffffffffu, t_max, o));
          // t_max up in [32, 64), or up = 2^127, the largest power of two
          float up_now = up;
          if (t_max > 0.f) up_now = fminf(up, __int_as_float((127 + min(5 + 127 - (__float_as_int(t_max) >> 23), 127)) << 23));
          const float scale_now = up_now / up;
          up = up_now;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float f[2], down[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float v = fmaxf(s[nt][e], s[nt][2 + e]);
              v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
              v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
              v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
              // (a query that sees nothing of the warp's first tile sees nothing of the later ones)
              const float d = begins ? (v == -INFINITY ? 0.f : v) : fmaxf(v, 0.f);
              f[e] = begins ? 0.f : ex2(-d);  // (the sums are still 0, and the first maximum may be far below it: no 0 inf)
              down[e] = d;
              s[nt][e] -= d, s[nt][2 + e] -= d;
            }
            m[nt] = add2(m[nt], two(-down[0], -down[1]));
            l[nt] = mul2(l[nt], two(f[0], f[1]));
            y[nt] = mul2(y[nt], two(f[0], f[1]));
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              f[e] *= scale_now;
              if (kSpare) {
                const float of_query = __shfl_xor_sync(0xffffffffu, f[e], 2);
                if (rests) f[e] = of_query;
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
              for (int mt = 0; mt < 8; ++mt) acc[mt][nt][e] *= f[e & 1];
            }
          }
        }

        // weights, and the second product
        uint32_t pb[NT][2], pr[NT][2];  // in two halves: rounded to fp16, and what that leaves
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float w_of = r ? -t_of[r] * up : t_of[r] * up;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const Two p = two(ex2(s[nt][2 * r]), ex2(s[nt][2 * r + 1]));
            l[nt] = add2(l[nt], p);
            y[nt] = fma2(p, two(y_of[r], y_of[r]), y[nt]);
            const float2 w = each(mul2(p, two(w_of, w_of)));
            uint2 halves = halves_f16(w.x, w.y);
            if (kSpare) {
              const uint32_t of_query = __shfl_xor_sync(0xffffffffu, halves.y, 2);
              if (rests) halves.x = of_query;
            } else {
              pr[nt][r] = transpose8(halves.y);
            }
            pb[nt][r] = transpose8(halves.x);
          }
        }
        // V rows of positions 2 t, 2 t + 1, 2 t + 8, 2 t + 9 of the tile, 8 bytes to a lane
        const uint32_t v_row = stage + (kChunk + h2 * 16 + t) * kKv4Row + ((g * 8) ^ ((t & 2) << 4));
        const uint2 v[4] = {lds64(v_row), lds64(v_row + 4 * kKv4Row), lds64(v_row + 8 * kKv4Row), lds64(v_row + 12 * kKv4Row)};
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
              const uint32_t z0 = hi ? x0 >> 8 : x0, z1 = hi ? x1 >> 8 : x1;
              const uint32_t a0 = z0 & 0x000f000fu, a1 = z0 & 0x00f000f0u, a2 = ~z1 & 0x000f000fu, a3 = ~z1 & 0x00f000f0u;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma_f16(acc[mt][nt], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
              if (!kSpare) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_f16(acc[mt][nt], a0, a1, a2, a3, pr[nt][0], pr[nt][1]);
              }
            }
          }
      }
    }
    cp_wait<0>();
    __syncthreads();  // the rings are free

    // ---- the warps' parts meet ----
    float* meet = reinterpret_cast<float*>(smem + K::kQBytes);
    {
      if (kSpare) {  // (the other columns' records are nobody's)
#pragma unroll
        for (int mt = 0; mt < 8; ++mt)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[mt][0][e] += __shfl_xor_sync(0xffffffffu, acc[mt][0][e], 2);
      }
      const float down = 1.f / up;  // (0 where the warp has seen nothing: its sums are 0)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float ls = e ? each(l[nt]).y : each(l[nt]).x, ys = e ? each(y[nt]).y : each(y[nt]).x;
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) {
            ls += __shfl_xor_sync(0xffffffffu, ls, o);
            ys += __shfl_xor_sync(0xffffffffu, ys, o);
          }
          float* rec = meet + (warp * K::kQueries + nt * 8 + 2 * t + e) * kRowFloats;
          if (g == 0) rec[kKv4D] = ls == 0.f ? -FLT_MAX : -(e ? each(m[nt]).y : each(m[nt]).x), rec[kKv4D + 1] = ls;
          // lane g has elements 16 g ... 16 g + 15: tile mt holds 2 mt (codes in the low half of a byte) and 2 mt + 1
#pragma unroll
          for (int mt = 0; mt < 8; mt += 2) {
            float4 o4;
            o4.x = fmaf(acc[mt][nt][e] * 16777216.f, down, ys);
            o4.y = fmaf(acc[mt][nt][2 + e] * 1048576.f, down, ys);
            o4.z = fmaf(acc[mt + 1][nt][e] * 16777216.f, down, ys);
            o4.w = fmaf(acc[mt + 1][nt][2 + e] * 1048576.f, down, ys);
            *reinterpret_cast<float4*>(rec + 16 * g + 2 * mt) = o4;
          }
        }
    }
    __syncthreads();
    const bool whole = seg0 == 0 && seg1 == n_chunks;
    float* rec = P.partial + static_cast<long long>(2 * blockIdx.x + (seg0 == 0 ? 1 : 0)) * units.rows * kRowFloats;
    finish<NWARP, NWARP, K::kQueries>(P, meet, b, h, row0, n_rows, whole, rec);
    if (tid == 0) {
      if (whole)
        P.flags[u] = S.bad[turn];
      else
        rec[kKv4D + 2] = __int_as_float(S.bad[turn]);
    }
    turn ^= 1;
    __syncthreads();  // the records have been read
    at = u_start + seg1;
    if (seg1 == n_chunks) {
      at = u_start += n_chunks + part.between;
      do {
        ++u;
      } while (u < units.n && at < last && chunks_of(P, u, kChunk) == 0);
    }
  }
}

}  // namespace
}  // namespace specattn
