// The path of specattn_kv4_verify on tcgen05, for 25 to 48 query rows.
//
// mma.sync does 1024 multiply-adds a cycle and SM, which 24 query rows use up at the speed of the memory; tcgen05 does
// four times that, and its operands need not pass through registers.  As in the bf16 kernel both products are taken
// transposed, with 128 positions (or the 128 elements of an output row) as the M side and N = 48 query rows (40 and zeros,
// say) as the other:
//     S^T [128 positions x N] = C_K [128 x 128] Q^T            C_K in tensor memory, Q in shared memory
//     O^T [128 elements x 80] += (C_V - m)^T [128 x 128] W     both in shared memory, position-major; 40 columns of the weights'
//                                                              first halves, 40 of their second: V is read once for both
// Two threads own a position, each half of its codes and half of the queries: they unpack the K row's codes by masks (the
// subnormals of fp16, see kv4_verify.cu) straight into their lane of tensor memory, and the V row's into a row of the
// swizzled operand; they get the position's scores back as that lane of S^T, so that scale and zero point are the
// threads' own; and they write the position's row of W.
// m, 8 and 7 in turn, tile by tile, is taken off the V codes by a packed subtraction, exact in fp16: the accumulators stay near zero
// instead of growing with the sum of the weights.  (The units cut off towards zero as they add; with 8 alone, half a code from the
// middle, 131072 positions came out 1.2e-4 of their size too large.)
//
// Two groups of eight warps take tiles of 128 positions in turn, each with operands, accumulators and a running maximum of
// its own, and run a phase apart.  In a group's turn:
//     scores of tile i from tensor memory | K of tile i + 1 into it | vote (may the maximum stay?) and S^T of i + 1 starts |
//     V of tile i, copies of tile i + 2 asked for | weights of tile i | O^T of tile i starts
// 40 rows over 8 x 8 x 32768 positions: 172 us, 1.7 TB/s.  A tile takes an SM about 2900 cycles, where HBM would take 757 and
// shared memory (16 KB of copies written and read, 32 KB of V operand, W and Q) about 1000: what bounds it is the chain of
// instructions, barriers and products in flight in a group's turn.  (A product each for the weights' two parts instead
// of one of 80 columns: 198 against 180 us.)
#pragma once
#include "kv4_verify.cuh"

namespace specattn {
namespace {

constexpr int kTile = 128;
constexpr int kTcWarps = 16;
constexpr int kTcRing = 2;
constexpr int kTcStage = kChunk * kKv4Row;  // half rows of K and V for 32 positions
constexpr int kTcSmem = 2 * 32768 + 4 * 16384 + 16384 + kTcWarps * kTcRing * kTcStage + 1024;

struct Tc4Shared {
  alignas(8) unsigned long long s_bar[2], o_bar[2];
  alignas(16) float4 base[2][32];  // of two of a group's queries: sums q, minus the running maxima
  float red[2][4][64][2];          // what the warps of a group reduce
  float t_red[2][4];
  float sums[2][64];  // sum of p (y + m t)
  float qsum[64];
  int limit[64];
  int bad[2], qmax[2];  // of this segment, and cleared for the next
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
// One thread of the warp, chosen by the hardware.  (Behind a branch on a thread's number descriptors go through vector
// registers: 8 products of 128 x 48 x 16 from tensor memory then take 760 cycles to issue and finish instead of 390.)
__device__ __forceinline__ bool elect() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void mma_smem(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(shape), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(shape), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void mma_done(unsigned long long* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tm_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// (the values pass through, so that nothing that uses them moves ahead of the wait)
__device__ __forceinline__ void tm_wait_ld4(float* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3])::"memory");
}
__device__ __forceinline__ void tm_pass4(float* r) {  // (for the values of a wait that has been made)
  asm volatile("" : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3])::"memory");
}
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_ld4(float* r, uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];" : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]) : "r"(at));
}
__device__ __forceinline__ void tm_st4(uint32_t at, const float* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]) : "memory");
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
__device__ __forceinline__ void sts64(uint32_t at, uint32_t a, uint32_t b) {
  asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(at), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ uint32_t minus(uint32_t a, uint32_t b) {
  const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}

// The 32 lanes' values of four columns, reduced: lane l gets column l & 3's.
template <typename Op>
__device__ __forceinline__ float of_four(const float* in, int lane, Op op) {
  float x[4] = {in[0], in[1], in[2], in[3]};
#pragma unroll
  for (int o = 2; o > 0; o >>= 1) {
    const bool upper = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float keep = upper ? x[i + o] : x[i], give = upper ? x[i] : x[i + o];
      x[i] = op(keep, __shfl_xor_sync(0xffffffffu, give, o));
    }
  }
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) x[0] = op(x[0], __shfl_xor_sync(0xffffffffu, x[0], o));
  return x[0];
}

template <int R8>
__device__ __forceinline__ void tc_path(const Kv4Params& P, const Partition& part, unsigned char* smem_raw, Tc4Shared& S) {
  constexpr int R = R8 * 8, CR = R / 2;                     // query rows; a thread's
  constexpr int N = (R8 + 1) / 2 * 16, NO = 2 * R;         // columns of the first product; of the second: rounded weights, then their remainders
  const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
  // group; half of a row's codes and of the queries; quarter of a tile; position of a tile = lane of tensor memory
  const int g = warp >> 3, half = (warp >> 2) & 1, wq = warp & 3, key = wq * 32 + lane, col0 = half * CR;
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t v_at = smem_u32(smem) + g * 32768, w_at = smem_u32(smem) + 65536 + g * 32768, q_at = smem_u32(smem) + 131072;
  const uint32_t ring_at = q_at + 16384 + warp * kTcRing * kTcStage;
  const Units units = units_of(P);

  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&S.tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&S.s_bar[i], 1);
      mbar_init(&S.o_bar[i], 1);
      S.bad[i] = S.qmax[i] = 0;
    }
    mbar_fence_init();
    S.abort = 0;
  }
  // (rows of Q beyond the query rows stay zero)
  for (int i = tid; i < 16384 / 16; i += kTcWarps * 32) reinterpret_cast<uint4*>(smem + 131072)[i] = make_uint4(0u, 0u, 0u, 0u);
  tm_before();
  __syncthreads();
  tm_after();
  const uint32_t tm_a = static_cast<uint32_t>(uniform(S.tmem)) + g * 256, tm_s = tm_a + 64, tm_o = tm_a + 128, mine = static_cast<uint32_t>(wq * 32) << 16;
  const uint64_t q_op = operand(q_at, 16, 1024), v_op = operand(v_at, kTile * 128, 1024), w_op = operand(w_at, 16384, 1024);
  const bool issues = (warp & 7) == 0;  // a warp of each group
  // where this thread's position has its weight for a column (W: 64 columns to a row of 128 bytes, pieces swizzled)
  auto weight_at = [&](int col) {
    return w_at + (col >> 6) * 16384 + key * 128 + ((((col & 63) >> 3) ^ (key & 7)) << 4) + (col & 4) * 2;
  };
  uint32_t s_turn = 0, o_turn = 0;  // completions of this group's products that have been waited for
  auto wait_for = [&](unsigned long long* bar, uint32_t turn) {
    if (!mbar_wait(bar, turn & 1u, &S.abort)) S.abort = 1;
  };
  const uint32_t swap = ((lane >> 2) & 1) << 4;  // raw half rows of 32 bytes: halves swapped so that 8 lanes meet all banks

  const int last = uniform(part.last);
  int u = uniform(part.unit), u_start = uniform(part.start), turn = 0;
  int b = 0, h = 0, seg0 = 0, seg1 = 0, n_tiles = 0, n_mine = 0, n_list = 0;
  int pos_next = 0, pg_next = -2, pos_then = 0;  // of this group's tile i + 2, of the one behind it
  uint32_t par_at = ~0u;                           // where its scales lie: of tile i + 1
  uint2 par;                                       // (s, z), (t, y) of this thread's position in the next tile
  auto index = [&](int i) { return (seg0 + g + 2 * i) * kTile + key; };  // in the unit, of this thread's position in the group's tile i
  auto position = [&](const Gather& G, int i) { return i < n_mine ? G.position(index(i)) : 0; };
  auto page = [&](const Gather& G, int i, int pos) { return i < n_mine ? G.page(index(i), pos) : -2; };
  // the warp copies its halves of 32 rows to a stage, K then V, two lanes to a row; the scales' place is returned, ~0: none
  auto fetch = [&](const Gather& G, int i, int pos, int pg) -> uint32_t {
    const uint32_t stage = ring_at + (i % kTcRing) * kTcStage;
    const uint2 row_at = G.locate(index(i), pos, pg, &S.bad[turn]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = j * 16 + (lane >> 1);
      const unsigned char* from = G.code_row(__shfl_sync(0xffffffffu, row_at.x, row) + half * 2 + (lane & 1));
      const uint32_t to = stage + row * 32 + (((lane & 1) ^ ((row >> 2) & 1)) << 4);
      cp_async16(to, from);
      cp_async16(to + kChunk * 32, from + P.cache.s_kv);
    }
    return index(i) < G.n_all ? row_at.y : ~0u;
  };
  auto scales = [&](const Gather& G, uint32_t place) {  // (zeros where there is no position)
    uint2 x = make_uint2(0u, 0u);
    if (place != ~0u) {
      const unsigned char* from = G.param_row(place);
      x.x = *reinterpret_cast<const uint32_t*>(from);
      x.y = *reinterpret_cast<const uint32_t*>(from + P.cache.p_kv);
    }
    return x;
  };
  // a segment's first tiles, asked for before the segment in front is finished
  auto begin = [&](int at) {
    b = u / P.H;
    h = u - b * P.H;
    const Gather G(P, b, h);
    n_list = G.n_list;
    n_tiles = (G.n_all + kTile - 1) / kTile;
    seg0 = at - u_start;
    seg1 = min(n_tiles, last - u_start);
    n_mine = max(0, (seg1 - seg0 - g + 1) >> 1);  // tiles seg0 + g, seg0 + g + 2, ...
    int pos[kTcRing + 2], pg[kTcRing + 1];
#pragma unroll
    for (int s = 0; s < kTcRing + 2; ++s) pos[s] = position(G, s);
#pragma unroll
    for (int s = 0; s < kTcRing + 1; ++s) pg[s] = page(G, s, pos[s]);
    par_at = ~0u;
    if (0 < n_mine) par = scales(G, fetch(G, 0, pos[0], pg[0]));
    cp_commit();
    if (1 < n_mine) par_at = fetch(G, 1, pos[1], pg[1]);
    cp_commit();
    pos_next = pos[2];
    pg_next = pg[2];
    pos_then = pos[3];
  };
  const int start_at = uniform(part.first);
  if (start_at < last) begin(start_at);

  for (int at = start_at; at < last;) {
    // ---- queries ----
    {
      Queries<kTcWarps, R> queries;
      queries.load(P, b, h, 0, P.rows);
      queries.look(P, 0, P.rows, &S.qmax[turn], S.qsum, S.limit);
      __syncthreads();
      const int qexp = query_exponent(S.qmax[turn]);
      queries.place(P, __int_as_float((127 + qexp) << 23),
                    [&](int r, int word, int part8, uint2 x) { sts64(q_at + swizzled(r, word, N) + part8 * 8, x.x, x.y); });
      if (tid < R) S.base[tid / CR][tid % CR] = make_float4(S.qsum[tid % CR * 2], S.qsum[tid % CR * 2 + 1], 0.f, 0.f);
      if (tid == 0) S.bad[turn ^ 1] = S.qmax[turn ^ 1] = 0;
      fence_proxy_async();
      __syncthreads();
    }
    const float k_mul = P.scale * 16777216.f * __int_as_float((127 - query_exponent(S.qmax[turn])) << 23);
    const Gather G(P, b, h);
    Two l[CR / 2], z[CR / 2];  // of two queries: sum of p, sum of p (y + m t) of this thread's positions
    float up = 3e38f;          // the weights' power of two: w = p t up
#pragma unroll
    for (int r = 0; r < CR / 2; ++r) l[r] = z[r] = two(0.f, 0.f);

    // half of the K codes of a stage's rows into tensor memory: two to a column, as the masks leave them
    auto k_codes = [&](int i) {
      const uint32_t row = ring_at + (i % kTcRing) * kTcStage + lane * 32;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint4 x = lds128(row + ((c << 4) ^ swap));
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        uint32_t a[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t v = w[j] >> 8;
          a[4 * j] = w[j] & 0x000f000fu, a[4 * j + 1] = w[j] & 0x00f000f0u;
          a[4 * j + 2] = v & 0x000f000fu, a[4 * j + 3] = v & 0x00f000f0u;
        }
        tm_st16(tm_a + mine + half * 32 + 16 * c, a);
      }
      tm_wait_st();
    };
    auto start_scores = [&](bool lost) {  // by one thread, after the barrier behind k_codes
      tm_after();
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
        mma_tmem(tm_s, tm_a + kk * 8, q_op + ((kk >> 2) * (N * 128) + (kk & 3) * 32) / 16, shape_word(N, 0), kk > 0);
      if (!lost) mma_done(&S.s_bar[g]);
    };
    if (n_mine > 0) {
      cp_wait<kTcRing - 1>();
      __syncwarp();
      k_codes(0);
      tm_before();
      named_bar_sync(1 + g, 256);
      // (test hook: the first scores of CTA 0 are never reported, so the bounded waits run out)
      if (issues && elect()) start_scores(P.test_lose && blockIdx.x == 0 && at == start_at);
      __syncwarp();
    }

#pragma unroll 1
    for (int i = 0; i < n_mine; ++i) {
      const uint32_t stage = ring_at + (i % kTcRing) * kTcStage;
      const bool more = i + 1 < n_mine;
      const float2 kp = widen16(par.x, P.half), vp = widen16(par.y, P.half);
      par = scales(G, par_at);  // of the next tile
      float x[CR];
      wait_for(&S.s_bar[g], s_turn++);
      tm_after();
#pragma unroll
      for (int c = 0; c < CR; c += 4) tm_ld4(x + c, tm_s + mine + col0 + c);
      if (more) {
        cp_wait<kTcRing - 2>();
        __syncwarp();
        k_codes(i + 1);
      }
      tm_wait_ld4(x);
#pragma unroll
      for (int c = 4; c < CR; c += 4) tm_pass4(x + c);
      // scores from the running maximum on
      const float ks = kp.x * k_mul;
      float t = vp.x, y8 = fmaf(i & 1 ? 7.f : 8.f, vp.x, vp.y), top = -INFINITY;
      const float4* base = S.base[g] + col0 / 2;
#pragma unroll
      for (int r = 0; r < CR; r += 2) {
        const float4 qm = base[r >> 1];
        const float2 x2 = each(fma2(two(x[r], x[r + 1]), two(ks, ks), fma2(two(kp.y, kp.y), two(qm.x, qm.y), two(qm.z, qm.w))));
        x[r] = x2.x, x[r + 1] = x2.y;
        top = fmaxf(top, fmaxf(x[r], x[r + 1]));
      }
      // what a query does not see: past the end, or behind it in the tail.  (A masked row may hold anything, and 0 NaN is
      // NaN: what a tail row's V scale would spoil, its scores spoil instead.)
      const int pos = index(i);
      if (__builtin_expect(pos - key + kTile > n_list, 0)) {
        const bool spoilt = pos >= n_list && !(fabsf(t) <= FLT_MAX && fabsf(y8) <= FLT_MAX);
        if (spoilt) t = y8 = 0.f;
        top = -INFINITY;
#pragma unroll
        for (int r = 0; r < CR; ++r) {
          if (spoilt) x[r] = NAN;
          if (pos >= n_list + S.limit[col0 + r]) x[r] = -INFINITY;
          top = fmaxf(top, x[r]);
        }
      }
      // the maximum moves only where a score passes it by 2^8, the weights' scale where one passes 64
      tm_before();
      const bool raise = named_bar_or(3 + g, 256, top > 8.f || fabsf(t) * up > 64.f || i == 0);
      if (issues && more && elect()) start_scores(false);
      __syncwarp();
      if (__builtin_expect(raise, 0)) {
        const auto larger = [](float a, float c) { return fmaxf(a, c); };
#pragma unroll
        for (int c = 0; c < CR; c += 4) {
          const float v = of_four(x + c, lane, larger);
          if (lane < 4) S.red[g][wq][col0 + c + lane][0] = v;
        }
        float t_max = fabsf(t) <= FLT_MAX ? fabsf(t) : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t_max = fmaxf(t_max, __shfl_xor_sync(0xffffffffu, t_max, o));
        if (lane == 0) S.t_red[g][wq] = t_max;
        named_bar_sync(1 + g, 256);
        t_max = fmaxf(fmaxf(S.t_red[g][0], S.t_red[g][1]), fmaxf(S.t_red[g][2], S.t_red[g][3]));
        float up_now = up;
        if (t_max > 0.f) up_now = fminf(up, __int_as_float((127 + min(5 + 127 - (__float_as_int(t_max) >> 23), 127)) << 23));
        const float scale_now = up_now / up;
        up = up_now;
        if (i > 0) {  // the output so far is complete, and has to shrink, too
          wait_for(&S.o_bar[g], o_turn);
          tm_after();
        }
#pragma unroll
        for (int c = 0; c < CR; c += 4) {
          float o[4], rest[4], f[4], down[4];
          if (i > 0) {
            tm_ld4(o, tm_o + mine + col0 + c);
            tm_ld4(rest, tm_o + mine + R + col0 + c);
            tm_wait_ld4(o);
            tm_pass4(rest);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = col0 + c + e;
            const float v = fmaxf(fmaxf(S.red[g][0][r][0], S.red[g][1][r][0]), fmaxf(S.red[g][2][r][0], S.red[g][3][r][0]));
            // (a query that sees nothing of the group's first tile sees nothing of the later ones)
            const float d = i == 0 ? (v == -INFINITY ? 0.f : v) : fmaxf(v, 0.f);
            f[e] = i == 0 ? 0.f : ex2(-d);  // (the sums are still 0, and the first maximum may be far below it: no 0 inf)
            x[c + e] -= d;
            o[e] *= f[e] * scale_now;
            rest[e] *= f[e] * scale_now;
            down[e] = d;
          }
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            l[(c + e) / 2] = mul2(l[(c + e) / 2], two(f[e], f[e + 1]));
            z[(c + e) / 2] = mul2(z[(c + e) / 2], two(f[e], f[e + 1]));
            if (key == (col0 + c + e) / 2) {
              float4& of = S.base[g][(col0 + c + e) / 2];
              of.z -= down[e];
              of.w -= down[e + 1];
            }
          }
          if (i > 0) tm_st4(tm_o + mine + col0 + c, o), tm_st4(tm_o + mine + R + col0 + c, rest);
        }
        tm_wait_st();
      }
      // the second product of the tile before has read V and W
      if (i > 0) {
        wait_for(&S.o_bar[g], o_turn++);
        tm_after();
      }
      {
        const uint32_t row = stage + (kChunk + lane) * 32, to = v_at + swizzled(key, 8 * half, kTile);
        const uint32_t mid = i & 1 ? 0x00070007u : 0x00080008u;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint4 raw = lds128(row + ((c << 4) ^ swap));
          const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t v = w[j] >> 8;
            sts128(to ^ ((4 * c + j) << 4), minus(w[j] & 0x000f000fu, mid), minus(w[j] & 0x00f000f0u, mid << 4),
                   minus(v & 0x000f000fu, mid), minus(v & 0x00f000f0u, mid << 4));
          }
        }
      }
      __syncwarp();  // the stage has been read
      par_at = i + kTcRing < n_mine ? fetch(G, i + kTcRing, pos_next, pg_next) : ~0u;
      cp_commit();
      pos_next = pos_then;
      pg_next = page(G, i + kTcRing + 1, pos_then);
      pos_then = position(G, i + kTcRing + 2);
      // weights
      const float w_of = t * up;
#pragma unroll
      for (int c = 0; c < CR; c += 4) {
        uint2 w[2];  // the halves of two each
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const Two p = two(ex2(x[c + e]), ex2(x[c + e + 1]));
          l[(c + e) / 2] = add2(l[(c + e) / 2], p);
          z[(c + e) / 2] = fma2(p, two(y8, y8), z[(c + e) / 2]);
          const float2 w2 = each(mul2(p, two(w_of, w_of)));
          w[e / 2] = halves_f16(w2.x, w2.y);
        }
        sts64(weight_at(col0 + c), w[0].x, w[1].x);
        sts64(weight_at(R + col0 + c), w[0].y, w[1].y);
      }
      fence_proxy_async();
      tm_before();
      named_bar_sync(1 + g, 256);
      if (issues && elect()) {
        tm_after();
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          mma_smem(tm_o, v_op + kk * 2048 / 16, w_op + kk * 2048 / 16, shape_word(NO, 1), kk > 0 ? 1 : i);
        mma_done(&S.o_bar[g]);
      }
      __syncwarp();
    }
    cp_wait<0>();

    // ---- the groups' parts meet ----
    const int this_u = u, this_b = b, this_h = h, this_mine = n_mine, this_turn = turn;
    const bool first_part = seg0 == 0, whole = seg0 == 0 && seg1 == n_tiles;
    at = u_start + seg1;
    if (seg1 == n_tiles) {
      at = u_start += n_tiles + part.between;
      do {
        ++u;
      } while (u < units.n && at < last && chunks_of(P, u, kTile) == 0);
    }
    turn ^= 1;
    if (at < last) begin(at);
    if (this_mine > 0) {
      wait_for(&S.o_bar[g], o_turn++);
      tm_after();
    }
    const auto add = [](float a, float c) { return a + c; };
#pragma unroll
    for (int c = 0; c < CR; c += 4) {
      const float2 l0 = each(l[c / 2]), l1 = each(l[c / 2 + 1]), z0 = each(z[c / 2]), z1 = each(z[c / 2 + 1]);
      const float l4[4] = {l0.x, l0.y, l1.x, l1.y}, z4[4] = {z0.x, z0.y, z1.x, z1.y};
      const float ls = of_four(l4, lane, add), zs = of_four(z4, lane, add);
      if (lane < 4) S.red[g][wq][col0 + c + lane][0] = ls, S.red[g][wq][col0 + c + lane][1] = zs;
    }
    __syncthreads();  // both groups are done with their operands: records take their place
    float* meet = reinterpret_cast<float*>(smem);
    static_assert(2 * R * kRowFloats * 4 <= 131072, "the spare rows of Q have to stay zero");
    if ((tid & 255) < R) {
      const int r = tid & 255;
      const float ls = (S.red[g][0][r][0] + S.red[g][1][r][0]) + (S.red[g][2][r][0] + S.red[g][3][r][0]);
      S.sums[g][r] = (S.red[g][0][r][1] + S.red[g][1][r][1]) + (S.red[g][2][r][1] + S.red[g][3][r][1]);
      float* rec = meet + (g * R + r) * kRowFloats;
      rec[kKv4D] = ls == 0.f ? -FLT_MAX : -(r & 1 ? S.base[g][r >> 1].w : S.base[g][r >> 1].z);
      rec[kKv4D + 1] = ls;
    }
    named_bar_sync(1 + g, 256);
    {
      // lane 8 i + j of O^T is element 8 i + (0, 4, 1, 5, 2, 6, 3, 7)[j], of the high half of a byte where j has bit 1
      const int j = key & 7, d = (key & ~7) + ((j & 1) << 2) + (j >> 1);
      const float down = (j & 2 ? 1048576.f : 16777216.f) / up;
#pragma unroll
      for (int c = 0; c < CR; c += 4) {
        float o[4], rest[4];
        if (this_mine > 0) {
          tm_ld4(o, tm_o + mine + col0 + c);
          tm_ld4(rest, tm_o + mine + R + col0 + c);
          tm_wait_ld4(o);
          tm_pass4(rest);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = col0 + c + e;
          meet[(g * R + r) * kRowFloats + d] = this_mine > 0 ? fmaf(o[e] + rest[e], down, S.sums[g][r]) : 0.f;
        }
      }
    }
    tm_before();
    __syncthreads();
    tm_after();
    float* rec = P.partial + static_cast<long long>(2 * blockIdx.x + (first_part ? 1 : 0)) * units.rows * kRowFloats;
    finish<kTcWarps, 2, R>(P, meet, this_b, this_h, 0, P.rows, whole, rec);
    if (tid == 0) {
      const int flag = S.bad[this_turn] | (S.abort ? SPECATTN_ROW_TIMEOUT : 0);
      if (whole)
        P.flags[this_u] = flag;
      else
        rec[kKv4D + 2] = __int_as_float(flag);
    }
    __syncthreads();  // the records have been read
  }
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(S.tmem), "r"(512u) : "memory");
}

}  // namespace
}  // namespace specattn
