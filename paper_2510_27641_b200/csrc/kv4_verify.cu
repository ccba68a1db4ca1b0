// specattn_kv4_verify: the attention of specattn_sparse_verify over a cache that holds its rows in 4 bits.
//
// The mathematics.  With K_i = s_i c_i + z_i and V_i = t_i e_i + y_i (codes c, e in 0..15),
//     q . K_i   = s_i (q . c_i) + z_i sum q
//     sum_i p_i V_i = sum_i (p_i t_i) (e_i - m) + sum_i p_i (y_i + m t_i)
// so both products run over the codes themselves (less an m that keeps the second's sums near zero) and the scales enter
// per (position, query) in binary32.  A code c as the bit pattern of an fp16 number is the subnormal c 2^-24, and 16 c is
// c 2^-20: masking a word of packed codes with 0x000f000f or 0x00f000f0 gives a register of two exact fp16 values and no
// conversion takes place (five instructions for eight codes; tensor cores take subnormals as they are).  Queries are scaled by a power of two so
// that they fit fp16 with all of their bits, those that meet the high codes of a byte by 2^-4 more.
// fp16 holds 11 bits of a weight w = p t, and sums of outputs in binary32 should not depend on so few: a weight goes in as
// two fp16 numbers, 21 bits, and the second product runs over both.  (With 11 bits alone 24 rows over 8 x 32768 took 122 us instead
// of 142, 40 rows 155 instead of 172; the outputs were off by 1e-4 to 5e-4 of their size, fp16 ones by half as much again as
// their own rounding.)
//
// Two paths compute this: on mma.sync (kv4_verify_mma.cuh) and, for 25 to 48 query rows, on tcgen05 (kv4_verify_tc.cuh).
// Units (sequence, KV head) are cut on the device, where the lengths are; the parts meet through the workspace in a second
// kernel, and nothing is held over from call to call.
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "kv4_verify.cuh"
#include "kv4_verify_mma.cuh"
#include "kv4_verify_tc.cuh"
#include "nvtx_range.h"

namespace specattn {

extern std::atomic<long long> g_launch_count;
int device_sm_count();

namespace {

// What a call of R8 * 8 query rows runs with.
//
// mma.sync: as many warps as hold a warp's output in registers.  Two groups of query rows, which read a unit's rows twice,
// from 33 rows on.
//
// tcgen05 takes 25 to 48 rows of calls over everything whose block table has room for least_chunks() chunks of 32 positions to an SM
// or more.  8 sequences x 8 heads, mma.sync against tcgen05:
//     x 32768   24 rows 142 / 143 us   28, 32 rows 170 / 155   40 rows 270 / 172   48 rows 270 / 199
//     x 4800 (65 chunks)  33.6 / 36.0             40.0 / 38.9         54.8 / 43.8           55.4 / 49.6
//     x 2400 (33 chunks)  23.0 / 25.7             27.0 / 27.6         33.3 / 31.5           33.3 / 35.5
//     x 1200              17.6 / 20.4             20.6 / 21.8         22.6 / 24.9           22.9 / 28.4
// (41 rows and more spill 200 bytes on tcgen05.)  Lists run on mma.sync, whatever room idx_stride gives them: their lengths are known
// on the device only, and a selection's stride is the context, of which it keeps a few per cent (40 rows, 4 x 8 lists with room
// for 131072: of 900 16.7 / 19.6 us, of 4000 32.4 / 32.7; only lists as long as 65536 lose, 256 / 167, and their caller may
// say so).  A kernel for each path: one for both, choosing by the lengths it found, cost small calls 3 us and 10 to 17 where
// the instructions were not in L2.
constexpr int least_chunks(int r8) { return r8 == 5 ? 32 : 64; }
template <int R8>  // (0: up to four rows)
struct Config {
  static constexpr bool kSpare = R8 == 0;
  static constexpr int kGroups = R8 > 4 ? 2 : 1;               // of query rows, on mma.sync: 32 are as many as registers hold
  static constexpr int kTiles = kSpare ? 1 : (R8 + kGroups - 1) / kGroups;  // of eight queries
  static constexpr bool kTensor = R8 >= 4 && R8 <= 6;
  static constexpr int kWarps = R8 <= 1 ? 16 : R8 == 2 ? 12 : 8;
  // Two chunks of 32 positions to a warp: one under way, one at work.  What the ring leaves is L1, where lists, tables and the
  // sectors of (s, z) pairs are met again (against three or four, with weights of 11 bits: 20 rows over 32 ragged lists 84
  // against 90 us, 4 rows over 16 ragged contexts 49 against 53, 24 rows over 8 x 32768 122 against 125).
  static constexpr int kStages = 2;
  using Mma = MmaPath<kTiles, kWarps, kStages>;
};

template <int R8>
__global__ void __launch_bounds__(Config<R8>::kWarps * 32, 1) kv4_verify_mma_kernel(const __grid_constant__ Kv4Params P) {
  using C = Config<R8>;
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ PartitionShared ps;
  __shared__ MmaShared<C::kTiles * 8> sh;
  pdl_wait();  // everything below reads what earlier kernels may have written
  if (threadIdx.x < 2) sh.bad[threadIdx.x] = sh.qmax[threadIdx.x] = 0;
  const Partition part = cut<C::kWarps * 32>(P, kChunk, C::kWarps, 32, ps);
  mma_path<C::kTiles, C::kWarps, C::kStages, C::kSpare>(P, part, smem, sh);
  pdl_launch_dependents();
}

template <int R8>
__global__ void __launch_bounds__(kTcWarps * 32, 1) kv4_verify_tc_kernel(const __grid_constant__ Kv4Params P) {
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ PartitionShared ps;
  __shared__ Tc4Shared sh;
  pdl_wait();
  const Partition part = cut<kTcWarps * 32>(P, kTile, 2, 12, ps);
  tc_path<R8>(P, part, smem, sh);
  pdl_launch_dependents();
}

// Joins the parts of units that several CTAs have worked on, and writes the rows of those that nobody has.
__global__ void __launch_bounds__(256) kv4_join_kernel(const __grid_constant__ Kv4Params P) {
  pdl_launch_dependents();
  pdl_wait();
  const Units units = units_of(P);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long rec_floats = static_cast<long long>(units.rows) * kRowFloats;
  // (the part of the CTA where a unit begins is that CTA's second record, all others are first records)
  auto rec_of = [&](int c, int first) { return P.partial + (2 * c + (c == first ? 1 : 0)) * rec_floats; };
  if (blockIdx.x == units.n) {  // the last block gathers the status words
    if (P.status == nullptr || blockIdx.y != 0) return;
    for (int b = warp; b < P.B; b += 8) {
      int flag = 0;
      for (int i = lane; i < units.n / P.B; i += 32) {
        const int u = (i / P.H) * P.B * P.H + b * P.H + i % P.H;
        const int2 of = P.parts[u];
        if (of.x == of.y) flag |= P.flags[u];
        if (of.x < of.y)
          for (int c = of.x; c <= of.y; ++c) flag |= __float_as_int(rec_of(c, of.x)[kKv4D + 2]);
      }
      flag = __reduce_or_sync(0xffffffffu, flag);
      if (lane == 0) P.status[b] = flag;
    }
    return;
  }
  const int u = blockIdx.x;
  const int2 of = P.parts[u];
  if (of.x == of.y) return;
  const int rg = u / (P.B * P.H), bh = u - rg * P.B * P.H, b = bh / P.H, h = bh - b * P.H;
  const int row0 = rg * units.rows, r = blockIdx.y * 8 + warp;
  if (r >= min(units.rows, P.rows - row0)) return;
  float m = -FLT_MAX, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  // four parts at a time, from a maximum that moves with them
  for (int c0 = of.x; c0 <= of.y; c0 += 4) {
    float2 ml[4];
    float4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      ml[j] = make_float2(-FLT_MAX, 0.f);
      x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (c0 + j <= of.y) {
        const float* rec = rec_of(c0 + j, of.x) + r * kRowFloats;
        ml[j] = *reinterpret_cast<const float2*>(rec + kKv4D);
        x[j] = *reinterpret_cast<const float4*>(rec + 4 * lane);
      }
    }
    const float top = fmaxf(m, fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x))), back = ex2(m - top);
    m = top;
    l *= back;
    o.x *= back, o.y *= back, o.z *= back, o.w *= back;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float f = ex2(ml[j].x - m);
      l = fmaf(f, ml[j].y, l);
      o.x = fmaf(f, x[j].x, o.x), o.y = fmaf(f, x[j].y, o.y), o.z = fmaf(f, x[j].z, o.z), o.w = fmaf(f, x[j].w, o.w);
    }
  }
  write_row(P, b, h, row0 + r, lane, o, m, l);
}

int query_tiles(const specattn_kv4_verify_args& A) { return (A.n_q * (A.n_q_heads / A.n_kv_heads) + 7) / 8; }
int groups_of(int r8) { return r8 > 4 ? 2 : 1; }

int validate(const specattn_kv4_verify_args* args) {
  if (args == nullptr) return SPECATTN_ERR_NULL;
  if (args->struct_size != sizeof(specattn_kv4_verify_args)) return SPECATTN_ERR_STRUCT_SIZE;
  const specattn_kv4_verify_args& A = *args;
  if (A.batch < 0 || A.n_q < 1 || A.n_q_heads < 1 || A.n_kv_heads < 1 || A.n_groups < 1 || A.n_q_heads % A.n_kv_heads != 0 ||
      (A.n_groups != 1 && A.n_groups != A.n_kv_heads) || !(A.sm_scale >= 0.f) || A.tail_len < 0 || A.tail_len > 64)
    return SPECATTN_ERR_RANGE;
  const int cc = kv4_check(A.cache);
  if (cc != SPECATTN_OK) return cc;
  if (A.cache.n_pages > INT32_MAX) return SPECATTN_ERR_RANGE;
  constexpr uint32_t kEngines = SPECATTN_VERIFY_ENGINE_MMA_SYNC | SPECATTN_VERIFY_ENGINE_TCGEN05;
  if ((A.flags & ~(kEngines | SPECATTN_VERIFY_TEST_LOSE_ARRIVAL)) != 0 || (A.flags & kEngines) == kEngines) return SPECATTN_ERR_RANGE;
  if (A.head_dim != kKv4D || A.n_q > SPECATTN_MAX_QUERY_ROWS || A.n_q_heads / A.n_kv_heads > SPECATTN_MAX_QUERY_ROWS / A.n_q ||
      static_cast<long long>(A.batch) * A.n_kv_heads > kMaxUnits)
    return SPECATTN_ERR_UNSUPPORTED;
  const int rows = A.n_q * (A.n_q_heads / A.n_kv_heads);
  if ((A.flags & SPECATTN_VERIFY_ENGINE_TCGEN05) && (rows <= 24 || rows > 48)) return SPECATTN_ERR_UNSUPPORTED;
  return SPECATTN_OK;
}

// parts, flags; then the records
size_t table_bytes(const specattn_kv4_verify_args& A) {
  return (static_cast<size_t>(A.batch) * A.n_kv_heads * groups_of(query_tiles(A)) * 3 + 63) / 64 * 256;
}
size_t workspace_bytes(const specattn_kv4_verify_args& A, int sms) {
  return table_bytes(A) + static_cast<size_t>(2) * sms * query_tiles(A) * 8 * kRowFloats * sizeof(float);
}

int launch_one(void (*kernel)(Kv4Params), const Kv4Params& P, dim3 grid, int threads, int smem, cudaStream_t stream) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, P) != cudaSuccess) {
    cudaGetLastError();
    return SPECATTN_ERR_CUDA;
  }
  g_launch_count.fetch_add(1, std::memory_order_relaxed);
  return SPECATTN_OK;
}

// most: the largest number of chunks of 32 positions that a call over everything can have, by its sizes
template <int R8>
int launch(Kv4Params& P, int engine, double most, int sms, cudaStream_t stream) {
  using C = Config<R8>;
  static std::atomic<unsigned long long> prepared{0};  // a bit per device
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return SPECATTN_ERR_CUDA;
  }
  if (!((prepared.load(std::memory_order_acquire) >> dev) & 1ull)) {
    cudaError_t rc = cudaFuncSetAttribute(kv4_verify_mma_kernel<R8>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::Mma::kSmem);
    if constexpr (C::kTensor)
      if (rc == cudaSuccess) rc = cudaFuncSetAttribute(kv4_verify_tc_kernel<R8>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTcSmem);
    if (rc != cudaSuccess) {
      cudaGetLastError();
      return SPECATTN_ERR_CUDA;
    }
    prepared.fetch_or(1ull << dev, std::memory_order_release);
  }
  P.n_units = P.B * P.H * C::kGroups;
  P.rows_per_unit = C::kTiles * 8;
  int rc = SPECATTN_OK;
  if constexpr (C::kTensor) {
    if (engine == 2 || (engine == 0 && P.dense && most >= static_cast<double>(least_chunks(R8)) * sms)) {
      P.n_units = P.B * P.H;
      P.rows_per_unit = R8 * 8;
      rc = launch_one(kv4_verify_tc_kernel<R8>, P, dim3(sms), kTcWarps * 32, kTcSmem, stream);
    } else {
      rc = launch_one(kv4_verify_mma_kernel<R8>, P, dim3(sms), C::kWarps * 32, C::Mma::kSmem, stream);
    }
  } else {
    rc = launch_one(kv4_verify_mma_kernel<R8>, P, dim3(sms), C::kWarps * 32, C::Mma::kSmem, stream);
  }
  if (rc != SPECATTN_OK) return rc;
  return launch_one(kv4_join_kernel, P, dim3(P.n_units + 1, C::kSpare ? 1 : R8), 256, 0, stream);
}

}  // namespace
}  // namespace specattn

extern "C" size_t specattn_kv4_verify_workspace_bytes(const specattn_kv4_verify_args* args) {
  if (specattn::validate(args) != SPECATTN_OK) return 0;
  const int sms = specattn::device_sm_count();
  if (sms <= 0) return 0;
  return specattn::workspace_bytes(*args, sms);
}

extern "C" int specattn_kv4_verify(const specattn_kv4_verify_args* args, void* cuda_stream) {
  using namespace specattn;
  NvtxRange nvtx_range("specattn_kv4_verify");
  const int v = validate(args);
  if (v != SPECATTN_OK) return v;
  const specattn_kv4_verify_args& A = *args;
  if (A.batch == 0) return SPECATTN_OK;
  if (!A.q || !A.kv_len || !A.out || !A.lse || !A.workspace) return SPECATTN_ERR_NULL;
  if (!A.dense && A.idx_stride < 0) return SPECATTN_ERR_RANGE;
  if (!A.dense && ((A.idx_stride > 0 && !A.idx) || !A.counts)) return SPECATTN_ERR_NULL;
  if ((!A.dense && A.idx_stride > kMaxPositions) ||
      (A.dense && A.cache.block_table_stride > kMaxPositions / A.cache.page_size))
    return SPECATTN_ERR_UNSUPPORTED;
  const int cb = kv4_check_buffers(A.cache);
  if (cb != SPECATTN_OK) return cb;
  if (reinterpret_cast<uintptr_t>(A.q) % 16 != 0 || reinterpret_cast<uintptr_t>(A.out) % 16 != 0 ||
      reinterpret_cast<uintptr_t>(A.workspace) % 256 != 0)
    return SPECATTN_ERR_ALIGN;
  const specattn_kv4_cache& cache = A.cache;
  // the kernel addresses codes in 16-byte and params in 4-byte units of 32 bits
  const double reach = (static_cast<double>(cache.n_pages) * cache.stride_page + cache.stride_kv +
                        static_cast<double>(cache.page_size) * cache.stride_slot) / 16;
  const double reach_params = (static_cast<double>(cache.n_pages) * cache.pstride_page + cache.pstride_kv +
                               static_cast<double>(cache.page_size) * cache.pstride_slot) / 2;
  if (cache.stride_page < 0 || cache.stride_kv < 0 || cache.stride_slot < 0 || cache.stride_head < 0 || cache.pstride_page < 0 ||
      cache.pstride_kv < 0 || cache.pstride_slot < 0 || cache.pstride_head < 0 || reach >= 4294967296. || reach_params >= 4294967296. ||
      cache.block_table_stride > INT32_MAX)
    return SPECATTN_ERR_UNSUPPORTED;
  const int sms = device_sm_count();
  if (sms <= 0) return SPECATTN_ERR_CUDA;
  if (A.workspace_bytes < workspace_bytes(A, sms)) return SPECATTN_ERR_WORKSPACE;
  const int r8 = query_tiles(A);
  Kv4Params P;
  memset(&P, 0, sizeof(P));
  P.cache = kv4_view(A.cache);
  P.c_page = static_cast<unsigned>(cache.stride_page / 16);
  P.c_slot = static_cast<unsigned>(cache.stride_slot / 16);
  P.p_page = static_cast<unsigned>(cache.pstride_page / 2);
  P.p_slot = static_cast<unsigned>(cache.pstride_slot / 2);
  P.pages_per_seq = static_cast<int>(cache.block_table_stride);
  P.q = static_cast<const unsigned char*>(A.q);
  P.kv_len = A.kv_len;
  P.idx = A.idx;
  P.counts = A.counts;
  P.idx_stride = A.idx_stride;
  P.out = static_cast<unsigned char*>(A.out);
  P.lse = A.lse;
  P.status = A.status;
  P.parts = static_cast<int2*>(A.workspace);
  P.flags = reinterpret_cast<int*>(P.parts + A.batch * A.n_kv_heads * groups_of(r8));
  P.partial = reinterpret_cast<float*>(static_cast<unsigned char*>(A.workspace) + table_bytes(A));
  P.scale = (A.sm_scale != 0.f ? A.sm_scale : 1.0f / sqrtf(static_cast<float>(A.head_dim))) * kLog2e;
  P.B = A.batch;
  P.T = A.n_q;
  P.Hq = A.n_q_heads;
  P.H = A.n_kv_heads;
  P.grp = A.n_q_heads / A.n_kv_heads;
  P.rows = A.n_q * P.grp;
  P.G = A.n_groups;
  P.dense = A.dense ? 1 : 0;
  P.tail = A.tail_len;
  P.out_f32 = A.out_f32 ? 1 : 0;
  P.half = A.cache.dtype == SPECATTN_DTYPE_FP16 ? 1 : 0;
  P.test_lose = A.flags & SPECATTN_VERIFY_TEST_LOSE_ARRIVAL ? 1 : 0;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const int engine = A.flags & SPECATTN_VERIFY_ENGINE_TCGEN05 ? 2 : A.flags & SPECATTN_VERIFY_ENGINE_MMA_SYNC ? 1 : 0;
  const double longest = static_cast<double>(cache.block_table_stride) * cache.page_size;
  const double most = static_cast<double>(A.batch) * A.n_kv_heads * ((longest + A.tail_len) / kChunk + 1);
  switch (P.rows <= 4 ? 0 : r8) {
    case 0: return launch<0>(P, engine, most, sms, stream);
    case 1: return launch<1>(P, engine, most, sms, stream);
    case 2: return launch<2>(P, engine, most, sms, stream);
    case 3: return launch<3>(P, engine, most, sms, stream);
    case 4: return launch<4>(P, engine, most, sms, stream);
    case 5: return launch<5>(P, engine, most, sms, stream);
    case 6: return launch<6>(P, engine, most, sms, stream);
    case 7: return launch<7>(P, engine, most, sms, stream);
    default: return launch<8>(P, engine, most, sms, stream);
  }
}
