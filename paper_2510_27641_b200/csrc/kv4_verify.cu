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
// The second product is taken about the middle of the codes: the weights w = p t are rounded to fp16, and an error of w
// should be multiplied by a code's distance from 8, not by the code (2 to 3 times the error of the output).
//
// Two paths compute this: on mma.sync (kv4_verify_mma.cuh) and on tcgen05 (kv4_verify_tc.cuh).  Which of them a call takes
// is decided on the device, where the lengths are: by every CTA alike, from the chunks of all units.  Units (sequence, KV
// head) are cut wherever the CTAs' equal shares end; the parts meet through the workspace in a second kernel, which
// holds nothing over from call to call.
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
// mma.sync: as many warps as hold a warp's output in registers.  tcgen05: sixteen warps of 128 registers, for 17 to 48 rows.
// Below, dequantising is all there is to do, and mma.sync does it with fewer steps (8 sequences x 8 heads x 32768 positions, 4
// / 16 query rows: 77 / 106 us against 119 / 126); above, sums do not fit (64 rows: 290 against 344).  Between, tcgen05 is
// ahead from `kTensorLeast` chunks of 32 positions to a CTA on (the same positions, 24 / 32 / 40 rows: 137 / 149 / 158 us
// against 145 / 168 / 249; 8 x 8 x 1200 positions, 16 chunks: 19.3 / 21.4 / 23.7 against 19.1 / 21.9 / 24.3).
template <int R8>
struct Config {
  static constexpr int kGroups = R8 > 4 ? 2 : 1;               // of query rows, on mma.sync: 32 are as many as registers hold
  static constexpr int kTiles = (R8 + kGroups - 1) / kGroups;  // of eight queries
  static constexpr bool kTensor = R8 >= 3 && R8 <= 6;
  static constexpr int kWarps = R8 == 1 ? 16 : R8 == 2 ? 12 : 8;
  static constexpr int kStages = R8 <= 2 ? 3 : 4;
  static constexpr int kThreads = kTensor ? kTcWarps * 32 : kWarps * 32;
  using Mma = MmaPath<kTiles, kWarps, kStages>;
  static constexpr int kSmem = kTensor && kTcSmem > Mma::kSmem ? kTcSmem : Mma::kSmem;
};
// Where both paths are there, a call on mma.sync gives eight of the sixteen warps' registers to the others.
constexpr int kLaunchRegisters = 128, kMoreRegisters = 232, kFewRegisters = 24;
static_assert(kMoreRegisters + kFewRegisters == 2 * kLaunchRegisters, "eight warps give what eight take");

template <int R8>
__global__ void __launch_bounds__(Config<R8>::kThreads, 1) kv4_verify_kernel(const __grid_constant__ Kv4Params P) {
  using C = Config<R8>;
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ PartitionShared ps;
  __shared__ union Shared {
    MmaShared<C::kTiles * 8> mma;
    Tc4Shared tc;
    __device__ Shared() {}
  } sh;
  pdl_wait();  // everything below reads what earlier kernels may have written
  if constexpr (C::kTensor) {
    constexpr int kTensorLeast = R8 == 3 ? 96 : R8 == 4 ? 0 : 16;
    bool tensor = P.engine == 2 || (P.engine == 0 && kTensorLeast == 0);
    if (P.engine == 0 && kTensorLeast > 0) {
      const int units = units_of(P, 1).n;
      int mine = 0, total;
      for (int u = threadIdx.x; u < units; u += C::kThreads) mine += chunks_of(P, u, kChunk);
      scan<C::kThreads>(mine, ps, &total);
      tensor = total >= kTensorLeast * static_cast<int>(gridDim.x);
    }
    if (tensor) {
      const Partition part = cut<C::kThreads>(P, 1, kTile, 2, 12, ps);
      tc_path<R8>(P, part, smem, sh.tc);
      pdl_launch_dependents();
      return;
    }
  }
  if (threadIdx.x < 2) sh.mma.bad[threadIdx.x] = sh.mma.qmax[threadIdx.x] = 0;
  const Partition part = cut<C::kThreads>(P, 0, kChunk, C::kWarps, 32, ps);
  if constexpr (C::kTensor) {
    if (threadIdx.x >= C::kWarps * 32) {
      set_max_registers_dec<kFewRegisters>();
      return;
    }
    set_max_registers_inc<kMoreRegisters>();
  }
  mma_path<C::kTiles, C::kWarps, C::kStages>(P, part, smem, sh.mma);
  pdl_launch_dependents();
}

// Joins the parts of units that several CTAs have worked on, and writes the rows of those that nobody has.
__global__ void __launch_bounds__(256) kv4_join_kernel(const __grid_constant__ Kv4Params P) {
  pdl_launch_dependents();
  pdl_wait();
  const Units units = units_of(P, *P.path);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long rec_floats = static_cast<long long>(units.rows) * kRowFloats;
  // (the part of the CTA where a unit begins is that CTA's second record, all others are first records)
  auto rec_of = [&](int c, int first) { return P.partial + (2 * c + (c == first ? 1 : 0)) * rec_floats; };
  if (blockIdx.x == P.most_units) {  // the last block gathers the status words
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
  if (u >= units.n) return;
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
  if (A.head_dim != kKv4D || A.n_q > SPECATTN_MAX_QUERY_ROWS || A.n_q * (A.n_q_heads / A.n_kv_heads) > SPECATTN_MAX_QUERY_ROWS ||
      static_cast<long long>(A.batch) * A.n_kv_heads > kMaxUnits)
    return SPECATTN_ERR_UNSUPPORTED;
  const int rows = A.n_q * (A.n_q_heads / A.n_kv_heads);
  if ((A.flags & SPECATTN_VERIFY_ENGINE_TCGEN05) && (rows <= 16 || rows > 48)) return SPECATTN_ERR_UNSUPPORTED;
  return SPECATTN_OK;
}

// the path, parts, flags; then the records
size_t table_bytes(const specattn_kv4_verify_args& A) {
  return (static_cast<size_t>(A.batch) * A.n_kv_heads * groups_of(query_tiles(A)) * 3 + 2 + 63) / 64 * 256;
}
size_t workspace_bytes(const specattn_kv4_verify_args& A, int sms) {
  return table_bytes(A) + static_cast<size_t>(2) * sms * query_tiles(A) * 8 * kRowFloats * sizeof(float);
}

template <int R8>
int launch(const Kv4Params& P, int sms, cudaStream_t stream) {
  using C = Config<R8>;
  static std::atomic<unsigned long long> prepared{0};  // a bit per device
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return SPECATTN_ERR_CUDA;
  }
  if (!((prepared.load(std::memory_order_acquire) >> dev) & 1ull)) {
    // (what one half of the warps gives the other takes: with fewer registers at launch they would wait for ever)
    cudaFuncAttributes built;
    if (cudaFuncGetAttributes(&built, kv4_verify_kernel<R8>) != cudaSuccess || (C::kTensor && built.numRegs != kLaunchRegisters) ||
        cudaFuncSetAttribute(kv4_verify_kernel<R8>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) != cudaSuccess) {
      cudaGetLastError();
      return SPECATTN_ERR_CUDA;
    }
    prepared.fetch_or(1ull << dev, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(sms);
  cfg.blockDim = dim3(C::kThreads);
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kv4_verify_kernel<R8>, P) != cudaSuccess) {
    cudaGetLastError();
    return SPECATTN_ERR_CUDA;
  }
  cfg.gridDim = dim3(P.most_units + 1, R8);
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = 0;
  if (cudaLaunchKernelEx(&cfg, kv4_join_kernel, P) != cudaSuccess) {
    cudaGetLastError();
    return SPECATTN_ERR_CUDA;
  }
  g_launch_count.fetch_add(2, std::memory_order_relaxed);
  return SPECATTN_OK;
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
  if (A.workspace_bytes < workspace_bytes(A, sms)) return SPECATTN_ERR_WORKSPACE;
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
  const int r8 = query_tiles(A), groups = groups_of(r8);
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
  P.most_units = A.batch * A.n_kv_heads * groups;
  P.path = static_cast<int*>(A.workspace);
  P.parts = reinterpret_cast<int2*>(P.path + 2);
  P.flags = P.path + 2 + 2 * P.most_units;
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
  P.engine = A.flags & SPECATTN_VERIFY_ENGINE_TCGEN05 ? 2 : A.flags & SPECATTN_VERIFY_ENGINE_MMA_SYNC ? 1 : 0;
  P.test_lose = A.flags & SPECATTN_VERIFY_TEST_LOSE_ARRIVAL ? 1 : 0;
  P.groups_of_rows = groups;
  P.rows_per_group = (r8 + groups - 1) / groups * 8;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  switch (r8) {
    case 1: return launch<1>(P, sms, stream);
    case 2: return launch<2>(P, sms, stream);
    case 3: return launch<3>(P, sms, stream);
    case 4: return launch<4>(P, sms, stream);
    case 5: return launch<5>(P, sms, stream);
    case 6: return launch<6>(P, sms, stream);
    case 7: return launch<7>(P, sms, stream);
    default: return launch<8>(P, sms, stream);
  }
}
