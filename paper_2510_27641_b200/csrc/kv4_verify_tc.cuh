// The path of specattn_kv4_verify on tcgen05, for 17 query rows and more over long lists.
//
// mma.sync does 1024 multiply-adds a cycle and SM, which 24 query rows use up at the speed of the memory; tcgen05 does
// four times that, and its operands need not pass through registers.  As in the bf16 kernel both products are taken
// transposed, with 128 positions (or the 128 elements of an output row) as the M side and the N = 32 ... 64 query rows
// as the other:
//     S^T [128 positions x N] = C_K [128 x 128] Q^T            C_K in tensor memory, Q in shared memory
//     O^T [128 elements x N] += (C_V - 8)^T [128 x 128] W      both in shared memory, position-major
// A thread owns a position: it unpacks the K row's codes by masks (the subnormals of fp16, see kv4_verify.cu) straight into
// its lane of tensor memory, and the V row's into a row of the swizzled operand; it gets the position's scores back
// as its lane of S^T, so that scale and zero point are the thread's own; and it writes the position's row of W.
// 8 is taken off the V codes by a packed subtraction, exact in fp16: the weights' rounding errors then multiply a
// code's distance from the middle, and the accumulators do not grow with the sum of the weights.
//
// Two groups of four warps take tiles of 128 positions in turn, each with operands, accumulators and a running maximum of
// its own, and run a phase apart.  In a group's turn:
//     scores of tile i from tensor memory | K of tile i + 1 into it | vote (may the maximum stay?) and S^T of i + 1 starts |
//     V of tile i | weights of tile i | O^T of tile i starts
// Shared memory takes 17 KB of copies, 16 KB of reads, 32 KB of V operand written and read each, and W and Q: about
// 940 cycles a tile at 128 bytes a cycle, where HBM takes 757 at 1.9 GHz.
#pragma once
#include "kv4_verify.cuh"

namespace specattn {
namespace {

constexpr int kTile = 128;
constexpr int kTcWarps = 8;
constexpr int kTcRing = 3;
constexpr int kTcSmem = 2 * 32768 + 2 * 16384 + 16384 + kTcWarps * kTcRing * kStageBytes + 1024;

struct Tc4Shared {
  alignas(8) unsigned long long s_bar[2], o_bar[2];
  alignas(16) float2 base[2][64];  // (sum q, minus the running maximum) of a group's queries
  float red[2][4][64][2];          // what the warps of a group reduce
  float t_red[2][4];
  float sums[2][64][2];            // sum of p, sum of p (y + 8 t)
  float qsum[64];
  int limit[64];
  int bad[2], qmax;
  uint32_t tmem;
  volatile int abort;
};

// byte offset of 16-byte piece c (0..15) of row r in an operand of `rows` rows of 256 bytes: two halves of 128 bytes,
// pieces swizzled by the row
__device__ __forceinline__ uint32_t swizzled(int r, int c, int rows) {
  return static_cast<uint32_t>((c >> 3) * rows * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t leading, uint32_t stride) {
  return static_cast<uint64_t>((at >> 4) & 0x3FFFu) | static_cast<uint64_t>((leading >> 4) & 0x3FFFu) << 16 |
         static_cast<uint64_t>((stride >> 4) & 0x3FFFu) << 32 | 1ull << 46 | 2ull << 61;
}
// fp16 x fp16 -> binary32, 128 x N, both operands K-major (0) or MN-major (1)
__device__ __forceinline__ uint32_t shape_word(int n, uint32_t mn_major) {
  return (1u << 4) | (mn_major << 15) | (mn_major << 16) | (static_cast<uint32_t>(n >> 3) << 17) | (8u << 24);
}
__device__ __forceinline__ void mma_smem(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5}, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(shape), "r"(acc), "r"(0u)
      : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %5, %5, %5}, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(shape), "r"(acc), "r"(0u)
      : "memory");
}
__device__ __forceinline__ void mma_done(unsigned long long* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tm_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// (the values pass through, so that nothing that uses them moves ahead of the wait)
__device__ __forceinline__ void tm_wait_ld8(float* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7])::"memory");
}
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_ld8(float* r, uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7])
               : "r"(at));
}
__device__ __forceinline__ void tm_st8(uint32_t at, const float* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(at), "f"(r[0]), "f"(r[1]),
               "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7])
               : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint32_t minus(uint32_t a, uint32_t b) {
  const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}

// The 32 lanes' values of eight columns, reduced: lane l gets column l & 7's.
template <typename Op>
__device__ __forceinline__ float of_eight(const float* in, int lane, Op op) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = in[i];
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) {
    const bool upper = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float keep = upper ? x[i + o] : x[i], give = upper ? x[i] : x[i + o];
      x[i] = op(keep, __shfl_xor_sync(0xffffffffu, give, o));
    }
  }
  x[0] = op(x[0], __shfl_xor_sync(0xffffffffu, x[0], 8));
  return op(x[0], __shfl_xor_sync(0xffffffffu, x[0], 16));
}

template <int R8>
__device__ __forceinline__ void tc_path(const Kv4Params& P, const Partition& part, unsigned char* smem_raw, Tc4Shared& S) {
  constexpr int R = R8 * 8, N = (R8 + 1) / 2 * 16;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = warp >> 2, wq = warp & 3, key = wq * 32 + lane;  // group, quarter of a tile, position of a tile = lane of tensor memory
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t v_at = smem_u32(smem) + g * 32768, w_at = smem_u32(smem) + 65536 + g * 16384, q_at = smem_u32(smem) + 98304;
  const uint32_t ring_at = q_at + 16384 + warp * kTcRing * kStageBytes;
  const Units units = units_of(P, 1);

  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&S.tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) mbar_init(&S.s_bar[i], 1), mbar_init(&S.o_bar[i], 1);
    mbar_fence_init();
    S.abort = 0;
  }
  // (columns of W beyond the query rows stay zero)
  for (int i = tid; i < 2048; i += kTcWarps * 32) reinterpret_cast<uint4*>(smem + 65536)[i] = make_uint4(0u, 0u, 0u, 0u);
  tm_before();
  __syncthreads();
  tm_after();
  const uint32_t tm_a = S.tmem + g * 192, tm_s = tm_a + 64, tm_o = tm_a + 128, mine = static_cast<uint32_t>(wq * 32) << 16;
  const bool elected = (tid & 127) == 0;
  uint32_t s_turn = 0, o_turn = 0;  // completions of this group's products that have been waited for
  auto wait_for = [&](unsigned long long* bar, uint32_t turn) {
    if (!mbar_wait(bar, turn & 1u, &S.abort)) S.abort = 1;
  };
  const int piece_of = (lane >> 1) & 3;  // raw rows: pieces of 16 bytes swapped so that 8 lanes meet 8 banks' groups

  int u = part.unit, u_start = part.start, turn = 0;
  for (int at = part.first; at < part.last;) {
    const int b = u / P.H, h = u - b * P.H;
    const Gather G(P, b, h);
    const int n_list = G.n_list, n_tiles = (G.n_all + kTile - 1) / kTile;
    const int seg0 = at - u_start, seg1 = min(n_tiles, part.last - u_start);
    const int n_mine = max(0, (seg1 - seg0 - g + 1) >> 1);  // tiles seg0 + g, seg0 + g + 2, ...
    auto position = [&](int i) { return i < n_mine ? G.position((seg0 + g + 2 * i) * kTile + key) : -1; };
    auto fetch = [&](int i, int pos, int pg) {
      const auto place = [](int row, int piece) { return row * kKv4Row + ((piece ^ ((row >> 1) & 3)) << 4); };
      G.fetch(ring_at + (i % kTcRing) * kStageBytes, pos, pg, lane, &S.bad[turn], place, place);
    };
    int pos_next, pg_next, pos_then;  // of this group's tile i + 3, of the one behind it
    {
      int pos[kTcRing + 2], pg[kTcRing + 1];
#pragma unroll
      for (int s = 0; s < kTcRing + 2; ++s) pos[s] = position(s);
#pragma unroll
      for (int s = 0; s < kTcRing + 1; ++s) pg[s] = G.page(pos[s]);
#pragma unroll
      for (int s = 0; s < kTcRing; ++s) {
        if (s < n_mine) fetch(s, pos[s], pg[s]);
        cp_commit();
      }
      pos_next = pos[kTcRing];
      pg_next = pg[kTcRing];
      pos_then = pos[kTcRing + 1];
    }

    // ---- queries ----
    if (tid == 0) S.qmax = 0;
    __syncthreads();
    if (tid == 0) S.bad[turn ^ 1] = 0;
    look_at_queries<kTcWarps, R>(P, b, h, 0, P.rows, &S.qmax, S.qsum, S.limit);
    __syncthreads();
    const int qexp = query_exponent(S.qmax);
    const float q_up = __int_as_float((127 + qexp) << 23);
    for (int i = tid; i < N * 16; i += kTcWarps * 32) {
      const int r = i >> 4, c = i & 15;
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (r < P.rows) x = query_word(P, query_at(P, b, h, r) + c * 8, q_up);
      sts128(q_at + swizzled(r, c, 64), x.x, x.y, x.z, x.w);
    }
    if (tid < 2 * R) S.base[tid / R][tid % R] = make_float2(S.qsum[tid % R], 0.f);
    fence_proxy_async();
    __syncthreads();
    const float k_mul = P.scale * 16777216.f * __int_as_float((127 - qexp) << 23);
    float l[R], z[R], up = 3e38f;  // sum of p, sum of p (y + 8 t) of this thread's positions; w = p t up
#pragma unroll
    for (int r = 0; r < R; ++r) l[r] = z[r] = 0.f;

    // K codes of a stage into tensor memory: two to a column, as the masks leave them
    auto k_codes = [&](int i) {
      const uint32_t row = ring_at + (i % kTcRing) * kStageBytes + lane * kKv4Row;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint4 x = lds128(row + ((c ^ piece_of) << 4));
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        uint32_t a[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t v = w[j] >> 8;
          a[4 * j] = w[j] & 0x000f000fu, a[4 * j + 1] = w[j] & 0x00f000f0u;
          a[4 * j + 2] = v & 0x000f000fu, a[4 * j + 3] = v & 0x00f000f0u;
        }
        tm_st16(tm_a + mine + 16 * c, a);
      }
      tm_wait_st();
    };
    auto start_scores = [&](bool lost) {  // by one thread, after the barrier behind k_codes
      tm_after();
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
        mma_tmem(tm_s, tm_a + kk * 8, operand(q_at + (kk >> 2) * (64 * 128) + (kk & 3) * 32, 16, 1024), shape_word(N, 0), kk > 0);
      if (!lost) mma_done(&S.s_bar[g]);
    };
    if (n_mine > 0) {
      cp_wait<kTcRing - 1>();
      __syncwarp();
      k_codes(0);
      tm_before();
      named_bar_sync(1 + g, 128);
      // (test hook: the first scores of CTA 0 are never reported, so the bounded waits run out)
      if (elected) start_scores(P.test_lose && blockIdx.x == 0 && at == part.first);
      __syncwarp();
    }

#pragma unroll 1
    for (int i = 0; i < n_mine; ++i) {
      const uint32_t stage = ring_at + (i % kTcRing) * kStageBytes;
      const bool more = i + 1 < n_mine;
      const uint2 par = lds64(stage + 2 * kChunk * kKv4Row + lane * 8);
      const float2 kp = widen16(par.x, P.half), vp = widen16(par.y, P.half);
      float x[R];
      wait_for(&S.s_bar[g], s_turn++);
      tm_after();
#pragma unroll
      for (int c = 0; c < R8; ++c) tm_ld8(x + 8 * c, tm_s + mine + 8 * c);
      if (more) {
        cp_wait<kTcRing - 2>();
        __syncwarp();
        k_codes(i + 1);
      }
#pragma unroll
      for (int c = 0; c < R8; ++c) tm_wait_ld8(x + 8 * c);
      // scores from the running maximum on
      const float ks = kp.x * k_mul;
      float t = vp.x, y8 = fmaf(8.f, vp.x, vp.y), top = -INFINITY;
      const float4* base = reinterpret_cast<const float4*>(S.base[g]);
#pragma unroll
      for (int r = 0; r < R; r += 2) {
        const float4 qm = base[r >> 1];
        x[r] = fmaf(x[r], ks, fmaf(kp.y, qm.x, qm.y));
        x[r + 1] = fmaf(x[r + 1], ks, fmaf(kp.y, qm.z, qm.w));
        top = fmaxf(top, fmaxf(x[r], x[r + 1]));
      }
      // what a query does not see: past the end, or behind it in the tail.  (A masked row may hold anything, and 0 NaN is
      // NaN: what a tail row's V scale would spoil, its scores spoil instead.)
      const int pos = (seg0 + g + 2 * i) * kTile + key;
      if ((seg0 + g + 2 * i + 1) * kTile > n_list) {
        const bool spoilt = pos >= n_list && !(fabsf(t) <= FLT_MAX && fabsf(y8) <= FLT_MAX);
        if (spoilt) t = y8 = 0.f;
        top = -INFINITY;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (spoilt) x[r] = NAN;
          if (pos >= n_list + S.limit[r]) x[r] = -INFINITY;
          top = fmaxf(top, x[r]);
        }
      }
      // the maximum moves only where a score passes it by 2^8, the weights' scale where one passes 64
      tm_before();
      const bool raise = named_bar_or(3 + g, 128, top > 8.f || fabsf(t) * up > 64.f || i == 0);
      if (elected && more) start_scores(false);
      __syncwarp();
      if (raise) {
        const auto larger = [](float a, float c) { return fmaxf(a, c); };
#pragma unroll
        for (int c = 0; c < R8; ++c) {
          const float v = of_eight(x + 8 * c, lane, larger);
          if (lane < 8) S.red[g][wq][8 * c + lane][0] = v;
        }
        float t_max = fabsf(t) <= FLT_MAX ? fabsf(t) : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t_max = fmaxf(t_max, __shfl_xor_sync(0xffffffffu, t_max, o));
        if (lane == 0) S.t_red[g][wq] = t_max;
        named_bar_sync(1 + g, 128);
        t_max = fmaxf(fmaxf(S.t_red[g][0], S.t_red[g][1]), fmaxf(S.t_red[g][2], S.t_red[g][3]));
        float up_now = up;
        if (t_max > 0.f) up_now = fminf(up, __int_as_float((127 + min(5 + 127 - (__float_as_int(t_max) >> 23), 100)) << 23));
        const float scale_now = up_now / up;
        up = up_now;
        if (i > 0) {  // the output so far is complete, and has to shrink, too
          wait_for(&S.o_bar[g], o_turn);
          tm_after();
        }
#pragma unroll
        for (int c = 0; c < R8; ++c) {
          float o[8];
          if (i > 0) {
            tm_ld8(o, tm_o + mine + 8 * c);
            tm_wait_ld8(o);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int r = 8 * c + e;
            const float v = fmaxf(fmaxf(S.red[g][0][r][0], S.red[g][1][r][0]), fmaxf(S.red[g][2][r][0], S.red[g][3][r][0]));
            // (a query that sees nothing of the group's first tile sees nothing of the later ones)
            const float d = i == 0 ? (v == -INFINITY ? 0.f : v) : fmaxf(v, 0.f);
            const float f = ex2(-d);
            x[r] -= d;
            l[r] *= f;
            z[r] *= f;
            o[e] *= f * scale_now;
            if ((tid & 127) == r) S.base[g][r].y -= d;
          }
          if (i > 0) tm_st8(tm_o + mine + 8 * c, o);
        }
        tm_wait_st();
      }
      // the second product of the tile before has read V and W
      if (i > 0) {
        wait_for(&S.o_bar[g], o_turn++);
        tm_after();
      }
      {
        const uint32_t row = stage + (kChunk + lane) * kKv4Row;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint4 raw = lds128(row + ((c ^ piece_of) << 4));
          const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t v = w[j] >> 8;
            sts128(v_at + swizzled(key, 4 * c + j, kTile), minus(w[j] & 0x000f000fu, 0x00080008u), minus(w[j] & 0x00f000f0u, 0x00800080u),
                   minus(v & 0x000f000fu, 0x00080008u), minus(v & 0x00f000f0u, 0x00800080u));
          }
        }
      }
      __syncwarp();  // the stage has been read
      if (i + kTcRing < n_mine) fetch(i + kTcRing, pos_next, pg_next);
      cp_commit();
      pos_next = pos_then;
      pg_next = G.page(pos_then);
      pos_then = position(i + kTcRing + 2);
      // weights
      const float w_of = t * up;
#pragma unroll
      for (int c = 0; c < R8; ++c) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 8 * c + 2 * e;
          const float p0 = ex2(x[r]), p1 = ex2(x[r + 1]);
          l[r] += p0, l[r + 1] += p1;
          z[r] = fmaf(p0, y8, z[r]), z[r + 1] = fmaf(p1, y8, z[r + 1]);
          w[e] = pack_f16(p0 * w_of, p1 * w_of);
        }
        sts128(w_at + key * 128 + ((c ^ (key & 7)) << 4), w[0], w[1], w[2], w[3]);
      }
      fence_proxy_async();
      tm_before();
      named_bar_sync(1 + g, 128);
      if (elected) {
        tm_after();
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          mma_smem(tm_o, operand(v_at + kk * 2048, kTile * 128, 1024), operand(w_at + kk * 2048, 16384, 1024), shape_word(N, 1), i > 0 || kk > 0);
        mma_done(&S.o_bar[g]);
      }
      __syncwarp();
    }
    cp_wait<0>();
    if (n_mine > 0) {
      wait_for(&S.o_bar[g], o_turn++);
      tm_after();
    }

    // ---- the groups' parts meet ----
    const auto add = [](float a, float c) { return a + c; };
#pragma unroll
    for (int c = 0; c < R8; ++c) {
      const float ls = of_eight(l + 8 * c, lane, add), zs = of_eight(z + 8 * c, lane, add);
      if (lane < 8) S.red[g][wq][8 * c + lane][0] = ls, S.red[g][wq][8 * c + lane][1] = zs;
    }
    __syncthreads();  // both groups are done with their operands: records take their place
    float* meet = reinterpret_cast<float*>(smem);
    static_assert(R8 % 2 == 0 || 2 * R * kRowFloats * 4 <= 65536, "the spare columns of W have to stay zero");
    if ((tid & 127) < R) {
      const int r = tid & 127;
      const float ls = (S.red[g][0][r][0] + S.red[g][1][r][0]) + (S.red[g][2][r][0] + S.red[g][3][r][0]);
      S.sums[g][r][1] = (S.red[g][0][r][1] + S.red[g][1][r][1]) + (S.red[g][2][r][1] + S.red[g][3][r][1]);
      float* rec = meet + (g * R + r) * kRowFloats;
      rec[kKv4D] = ls == 0.f ? -FLT_MAX : -S.base[g][r].y;
      rec[kKv4D + 1] = ls;
    }
    named_bar_sync(1 + g, 128);
    {
      // lane 8 i + j of O^T is element 8 i + (0, 4, 1, 5, 2, 6, 3, 7)[j], of the high half of a byte where j has bit 1
      const int j = key & 7, d = (key & ~7) + ((j & 1) << 2) + (j >> 1);
      const float down = (j & 2 ? 1048576.f : 16777216.f) / up;
#pragma unroll
      for (int c = 0; c < R8; ++c) {
        float o[8];
        if (n_mine > 0) {
          tm_ld8(o, tm_o + mine + 8 * c);
          tm_wait_ld8(o);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
          meet[(g * R + 8 * c + e) * kRowFloats + d] = n_mine > 0 ? fmaf(o[e], down, S.sums[g][8 * c + e][1]) : 0.f;
      }
    }
    tm_before();
    __syncthreads();
    tm_after();
    const bool whole = seg0 == 0 && seg1 == n_tiles;
    float* rec = P.partial + static_cast<long long>(2 * blockIdx.x + (seg0 == 0 ? 1 : 0)) * units.rows * kRowFloats;
    finish<kTcWarps, 2, R>(P, meet, b, h, 0, P.rows, whole, rec);
    if (tid == 0) {
      const int flag = S.bad[turn] | (S.abort ? SPECATTN_ROW_TIMEOUT : 0);
      if (whole)
        P.flags[u] = flag;
      else
        rec[kKv4D + 2] = __int_as_float(flag);
    }
    turn ^= 1;
    __syncthreads();  // the records have been read
    at = u_start + seg1;
    if (seg1 == n_tiles) {
      u_start += n_tiles;
      do {
        ++u;
      } while (u < units.n && at < part.last && chunks_of(P, u, kTile) == 0);
    }
  }
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(S.tmem), "r"(512u) : "memory");
}

}  // namespace
}  // namespace specattn
