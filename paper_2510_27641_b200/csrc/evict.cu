// specattn_accumulate, specattn_evict, specattn_move_rows: giving up the rows of a cache that have had the least
// attention.
//
//   accumulate  one read of the draft maps, bound by HBM: a thread sums four neighbouring positions over the rows of
//               (head, query) in binary64 (a conversion and an addition a value: 1/8 of the SM's binary64 rate at
//               HBM's speed).  Few positions are dealt to several threads each, by rows.  260 MB: 42 us, 6.2 TB/s.
//   evict       one list to a cluster of CTAs that hold its weights as ordered 32-bit keys in shared memory.  The
//               m-th largest key is found digit by digit (four of 8 bits) from histograms that the cluster adds
//               up; which slots stay then follows from comparisons, and their ranks from counts.  Bound by the
//               chain of passes and cluster barriers: 15 us for 8 lists of 32768, 46 for 32 of 131072 (with positions).
//   move_rows   copies of rows, bound by HBM: 1.04 GB read and written in 168 us, 6.2 TB/s.
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "kv4.cuh"
#include "nvtx_range.h"
#include "ptx.cuh"
#include "specattn.h"

namespace specattn {

extern std::atomic<long long> g_launch_count;
int device_sm_count();

namespace {

// ---- accumulate --------------------------------------------------------------------------------
constexpr int kAccThreads = 256;

struct AccParams {
  const float* probs[SPECATTN_MAX_DRAFT_LAYERS];
  const int* kv_len;
  const float* in;
  float* out;
  int* row_status;
  long long L_stride, score_stride;
  double decay;
  int B, H, gamma, G;
  unsigned char head[SPECATTN_MAX_DRAFT_HEADS];            // heads by group
  unsigned short first[SPECATTN_MAX_DRAFT_HEADS + 1];      // where a group's heads begin (grouped calls)
  int grouped;
};

// Grid: (positions, sequence x group, layer).  kSlices threads share four positions, each taking every kSlices-th
// row; their sums meet in shared memory in the order of the slices.  Without groups of heads one block writes the
// sum to all groups.
template <int kSlices>
__global__ void __launch_bounds__(kAccThreads) accumulate_kernel(const __grid_constant__ AccParams P) {
  constexpr int kQuads = kAccThreads / kSlices;
  __shared__ double part[kSlices > 1 ? (kSlices - 1) * kQuads * 4 : 1];
  __shared__ unsigned char part_bad[kSlices > 1 ? (kSlices - 1) * kQuads : 1];
  const int u = blockIdx.z;
  const float* probs = P.probs[u];
  if (probs == nullptr) return;
  const int b = P.grouped ? blockIdx.y / P.G : blockIdx.y, g = P.grouped ? blockIdx.y - b * P.G : 0;
  long long n = P.kv_len[b];
  n = min(n, min(P.L_stride, P.score_stride));
  const int quad = threadIdx.x % kQuads, slice = threadIdx.x / kQuads;
  const long long i0 = (static_cast<long long>(blockIdx.x) * kQuads + quad) * 4;
  if (static_cast<long long>(blockIdx.x) * kQuads * 4 >= n) return;
  const int h0 = P.grouped ? P.first[g] : 0, n_heads = P.grouped ? P.first[g + 1] - h0 : P.H;
  const int rows = n_heads * P.gamma;
  const bool live = i0 < n;
  double sum[4] = {0., 0., 0., 0.};
  unsigned bad = 0;
  if (live) {
    const float* base = probs + static_cast<long long>(b) * P.H * P.gamma * P.L_stride + i0;
    constexpr int kAhead = 8;
    for (int r0 = slice; r0 < rows; r0 += kSlices * kAhead) {
      float4 x[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int r = r0 + j * kSlices;
        if (r >= rows) continue;
        int row = r;
        if (P.grouped) {
          const int h = r / P.gamma;
          row = P.head[h0 + h] * P.gamma + (r - h * P.gamma);
        }
        x[j] = __ldcs(reinterpret_cast<const float4*>(base + row * P.L_stride));
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (r0 + j * kSlices >= rows) continue;
        const float v[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          bad |= (v[e] >= 0.f && v[e] <= FLT_MAX) ? 0u : 1u << e;
          sum[e] += static_cast<double>(v[e]);
        }
      }
    }
  }
  if (kSlices > 1) {
    if (slice > 0) {
#pragma unroll
      for (int e = 0; e < 4; ++e) part[((slice - 1) * 4 + e) * kQuads + quad] = sum[e];
      part_bad[(slice - 1) * kQuads + quad] = static_cast<unsigned char>(bad);
    }
    __syncthreads();
    if (slice > 0 || !live) return;
#pragma unroll
    for (int s = 0; s < kSlices - 1; ++s) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += part[(s * 4 + e) * kQuads + quad];
      bad |= part_bad[s * kQuads + quad];
    }
  } else if (!live) {
    return;
  }
  if (i0 + 4 > n) bad &= (1u << (n - i0)) - 1u;
  const int g_end = P.grouped ? g + 1 : P.G;
  for (int gg = g; gg < g_end; ++gg) {
    const long long list = (static_cast<long long>(u) * P.B + b) * P.G + gg;
    const float* in = P.in != nullptr ? P.in + list * P.score_stride + i0 : nullptr;
    float* out = P.out + list * P.score_stride + i0;
    if (bad != 0 && P.row_status != nullptr) atomicOr(P.row_status + list, SPECATTN_ROW_INVALID_PROB);
    const bool wide = i0 + 4 <= n && reinterpret_cast<uintptr_t>(out) % 16 == 0 &&
                      (in == nullptr || reinterpret_cast<uintptr_t>(in) % 16 == 0);
    float old[4] = {0.f, 0.f, 0.f, 0.f}, now[4];
    if (in != nullptr) {
      if (wide) {
        const float4 v = *reinterpret_cast<const float4*>(in);
        old[0] = v.x, old[1] = v.y, old[2] = v.z, old[3] = v.w;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (i0 + e < n) old[e] = in[e];
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      now[e] = (bad >> e) & 1u ? old[e] : static_cast<float>(__dadd_rn(__dmul_rn(P.decay, static_cast<double>(old[e])), sum[e]));
    if (wide) {
      *reinterpret_cast<float4*>(out) = make_float4(now[0], now[1], now[2], now[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (i0 + e < n) out[e] = now[e];
    }
  }
}

// ---- evict ---------------------------------------------------------------------------------------
constexpr int kEvBins = 256;
constexpr int kEvCopies = 8;  // of a histogram: weights share their leading bits, and lanes that meet in a bin wait for one another
constexpr int kEvMaxCluster = 8;
constexpr int kEvMaxSlice = SPECATTN_MAX_KV_LEN / kEvMaxCluster;  // keys of a CTA

struct EvictParams {
  const float* scores;
  const int *kv_len, *positions, *seq_len;
  int *src, *dst, *n_moves, *new_len;
  float* scores_out;
  int* positions_out;
  long long L, move_stride;
  int budget, n_sink, n_recent, B, G, slice;
  int wide;  // whether four neighbouring entries of every array may be read and written at once
};

struct EvictShared {
  alignas(16) unsigned hist[4][kEvBins * kEvCopies];  // one for each digit; copy c of bin d at d * kEvCopies + c
  unsigned sums[4][kEvBins];                          // of the copies, for the peers
  unsigned warp[33];
  unsigned found[3];  // digit, keys above it, keys at it
  unsigned count[2];  // of this CTA's slice: ties; stays behind the budget, and from bit 16 on gaps in front of it
};

// Larger weight, larger key; every key of a slot that exists is above 0, a protected slot's above all weights'.
__device__ __forceinline__ uint32_t key_of(float w) {
  if (w != w) w = -INFINITY;
  w += 0.f;  // -0 to 0
  const uint32_t u = __float_as_uint(w);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// The exclusive prefix of v over the threads of the CTA and its total.
template <int kThreads>
__device__ __forceinline__ unsigned block_prefix(unsigned v, unsigned* warp_sums, unsigned* total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  unsigned x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();  // the last call's sums have been read
  if (lane == 31) warp_sums[w] = x;
  __syncthreads();
  // (every warp adds up the others' for itself)
  unsigned t = lane < kThreads / 32 ? warp_sums[lane] : 0u;
  const unsigned mine = t;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, t, o);
    if (lane >= o) t += y;
  }
  *total = __shfl_sync(0xffffffffu, t, 31);
  return __shfl_sync(0xffffffffu, t - mine, w) + x - v;
}

__device__ __forceinline__ unsigned ld_peer(const unsigned* local, uint32_t rank) {
  unsigned v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_to_cta(smem_u32(local), rank)) : "memory");
  return v;
}

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
  return r;
}

__device__ __forceinline__ void cluster_sync() {
  cluster_arrive_release();
  cluster_wait();
}

// One list to a cluster.  Slots are dealt to the CTAs in slices and, within a slice, to warps in runs of 32, so that
// ranks in slot order are sums over runs: a thread that owns a run's lane learns its rank from the ballot, the runs in
// front of it in its warp's stretch, and the stretches in front of that.
template <int kEvThreads>
__global__ void __launch_bounds__(kEvThreads) evict_kernel(const __grid_constant__ EvictParams P) {
  constexpr int kEvWarps = kEvThreads / 32;
  extern __shared__ uint32_t keys[];
  __shared__ EvictShared S;
  const uint32_t rank = cluster_cta_rank(), n_cta = cluster_size();
  const long long list = blockIdx.x / n_cta;
  const int b = static_cast<int>((list / P.G) % P.B);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = static_cast<int>(max(0ll, min(static_cast<long long>(P.kv_len[b]), P.L)));
  const int m = min(n, P.budget);
  if (list < P.B * P.G && list % P.G == 0 && rank == 0 && tid == 0) P.new_len[b] = m;
  const float* scores = P.scores + list * P.L;
  const int* positions = P.positions != nullptr ? P.positions + list * P.L : nullptr;
  float* scores_out = P.scores_out != nullptr ? P.scores_out + list * P.L : nullptr;
  int* positions_out = P.positions_out != nullptr ? P.positions_out + list * P.L : nullptr;
  const int at = static_cast<int>(rank) * P.slice;  // first slot of this CTA
  const int mine = max(0, min(P.slice, n - at));
  const bool copy_scores = scores_out != nullptr && scores_out != scores;
  const bool copy_positions = positions_out != nullptr && positions_out != positions;
  for (int i = tid; i < kEvBins * kEvCopies; i += kEvThreads) reinterpret_cast<uint4*>(&S.hist[0][0])[i] = make_uint4(0u, 0u, 0u, 0u);
  __syncthreads();
  // keys, and the first digit's histogram; copies of what may stay where it is (moves overwrite the rest of it later)
  {
    const long long end = P.seq_len != nullptr ? P.seq_len[b] : n;
    const long long recent = end - P.n_recent;
    auto take = [&](int i, float w, int pos) {
      const uint32_t k = pos < P.n_sink || pos >= recent ? 0xffffffffu : key_of(w);
      keys[i] = k;
      atomicAdd(&S.hist[0][(k >> 24) * kEvCopies + (lane & (kEvCopies - 1))], 1u);
    };
    constexpr int kAhead = 2;  // quads of slots in flight to a thread
    const bool quads = P.wide && at % 4 == 0;
    const int whole = quads ? mine & ~3 : 0;
    for (int i0 = tid * 4; i0 < whole; i0 += kAhead * kEvThreads * 4) {
      float4 w[kAhead];
      int4 pos[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = i0 + j * kEvThreads * 4;
        if (i >= whole) continue;
        w[j] = *reinterpret_cast<const float4*>(scores + at + i);
        pos[j] = positions != nullptr ? *reinterpret_cast<const int4*>(positions + at + i) : make_int4(at + i, at + i + 1, at + i + 2, at + i + 3);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = i0 + j * kEvThreads * 4;
        if (i >= whole) continue;
        take(i, w[j].x, pos[j].x), take(i + 1, w[j].y, pos[j].y), take(i + 2, w[j].z, pos[j].z), take(i + 3, w[j].w, pos[j].w);
        const int front = m - (at + i);  // of the four, those that lie in front of the budget
        if (copy_scores)
          *reinterpret_cast<float4*>(scores_out + at + i) =
              make_float4(front > 0 ? w[j].x : 0.f, front > 1 ? w[j].y : 0.f, front > 2 ? w[j].z : 0.f, front > 3 ? w[j].w : 0.f);
        if (copy_positions) {
          if (front > 3) {
            *reinterpret_cast<int4*>(positions_out + at + i) = pos[j];
          } else {
            if (front > 0) positions_out[at + i] = pos[j].x;
            if (front > 1) positions_out[at + i + 1] = pos[j].y;
            if (front > 2) positions_out[at + i + 2] = pos[j].z;
          }
        }
      }
    }
    for (int i = whole + tid; i < mine; i += kEvThreads) {
      const float w = scores[at + i];
      const int pos = positions != nullptr ? positions[at + i] : at + i;
      take(i, w, pos);
      if (copy_scores) scores_out[at + i] = at + i < m ? w : 0.f;
      if (copy_positions && at + i < m) positions_out[at + i] = pos;
    }
  }
  if (n == m) {  // everything stays (the same for the whole cluster)
    if (rank == 0 && tid == 0) P.n_moves[list] = 0;
    return;
  }
  __syncthreads();

  // the m-th largest key: its digits, and how many of the keys equal to it stay
  uint32_t prefix = 0;  // the digits found so far
  unsigned want = static_cast<unsigned>(m), ties = 0;
#pragma unroll 1
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
    if (pass > 0) {
      const uint32_t above = 0xffffff00u << shift;
      unsigned* hist = S.hist[pass] + (lane & (kEvCopies - 1));
#pragma unroll 4
      for (int i = tid; i < mine; i += kEvThreads) {
        const uint32_t k = keys[i];
        if ((k & above) == prefix) atomicAdd(&hist[((k >> shift) & 255u) * kEvCopies], 1u);
      }
      __syncthreads();
    }
    if (tid < kEvBins) {
      const uint4 a = *reinterpret_cast<const uint4*>(&S.hist[pass][tid * kEvCopies]), b4 = *reinterpret_cast<const uint4*>(&S.hist[pass][tid * kEvCopies + 4]);
      S.sums[pass][tid] = (a.x + a.y + a.z + a.w) + (b4.x + b4.y + b4.z + b4.w);
    }
    cluster_sync();
    // every CTA adds up all histograms, the largest digits first
    const int digit = kEvBins - 1 - tid;
    unsigned c = 0;
    if (tid < kEvBins)
      for (uint32_t r = 0; r < n_cta; ++r) c += ld_peer(&S.sums[pass][digit], r);
    unsigned total;
    const unsigned run = block_prefix<kEvThreads>(c, S.warp, &total);
    if (run < want && run + c >= want) S.found[0] = static_cast<unsigned>(digit), S.found[1] = run, S.found[2] = c;
    __syncthreads();
    prefix |= S.found[0] << shift;
    want -= S.found[1];
    ties = S.found[2];
  }
  const uint32_t cut = prefix;  // slots above it stay, and the first `want` of the `ties` slots at it

  // each warp has a stretch of the slice
  const int stretch = ((P.slice + kEvWarps - 1) / kEvWarps + 31) / 32 * 32;
  const int w0 = min(warp * stretch, mine), w1 = min(w0 + stretch, mine);
  unsigned tie_rank = 0;  // of the first tie of this warp's stretch
  const bool split = want < ties;
  if (split) {
    unsigned t = 0;
    for (int i = w0 + lane; i < w1; i += 32) t += keys[i] == cut ? 1u : 0u;
    unsigned total;
    const unsigned before = block_prefix<kEvThreads>(t, S.warp, &total);
    if (tid == 0) S.count[0] = total;
    cluster_sync();
    tie_rank = __shfl_sync(0xffffffffu, before, 0);
    for (uint32_t r = 0; r < rank; ++r) tie_rank += ld_peer(&S.count[0], r);
  }
  auto ballots = [&](int i, unsigned* ties_so_far) {  // which of the 32 slots from i on stay
    const uint32_t k = i + lane < w1 ? keys[i + lane] : 0u;
    bool stays = k >= cut;
    if (split) {
      const unsigned at_cut = __ballot_sync(0xffffffffu, k == cut);
      if (k == cut) stays = *ties_so_far + __popc(at_cut & ((1u << lane) - 1u)) < want;
      *ties_so_far += __popc(at_cut);
    }
    return __ballot_sync(0xffffffffu, stays && i + lane < w1);
  };
  unsigned n_from = 0, n_into = 0, seen = tie_rank;
#pragma unroll 4
  for (int i = w0; i < w1; i += 32) {
    const unsigned stays = ballots(i, &seen);
    const unsigned exist = w1 - i >= 32 ? 0xffffffffu : (1u << (w1 - i)) - 1u;
    const int front = m - (at + i);  // slots in front of the budget
    const unsigned in_front = front >= 32 ? 0xffffffffu : front <= 0 ? 0u : (1u << front) - 1u;
    n_from += __popc(stays & ~in_front);
    n_into += __popc(exist & ~stays & in_front);
  }
  // (a slice has fewer than 2^16 slots: both counts in one word)
  unsigned total_both;
  const unsigned both = block_prefix<kEvThreads>(lane == 0 ? n_from | n_into << 16 : 0u, S.warp, &total_both);
  if (tid == 0) S.count[1] = total_both;
  cluster_sync();
  unsigned from = __shfl_sync(0xffffffffu, both, 0), into = from >> 16;
  from &= 0xffffu;
  for (uint32_t r = 0; r < rank; ++r) {
    const unsigned x = ld_peer(&S.count[1], r);
    from += x & 0xffffu;
    into += x >> 16;
  }
  // (the last thread's count is where the last slice ends)
  if (rank == n_cta - 1 && tid == kEvThreads - 1) P.n_moves[list] = static_cast<int>(from + n_from);

  // the lists, and what stays where it is
  int* src = P.src + list * P.move_stride;
  int* dst = P.dst + list * P.move_stride;
  seen = tie_rank;
#pragma unroll 4
  for (int i = w0; i < w1; i += 32) {
    const unsigned stays = ballots(i, &seen);
    const unsigned exist = w1 - i >= 32 ? 0xffffffffu : (1u << (w1 - i)) - 1u;
    const int slot = at + i + lane, front = m - (at + i);
    const unsigned in_front = front >= 32 ? 0xffffffffu : front <= 0 ? 0u : (1u << front) - 1u;
    const unsigned f = stays & ~in_front, t = exist & ~stays & in_front, low = (1u << lane) - 1u;
    if ((f >> lane) & 1u) src[from + __popc(f & low)] = slot;
    if ((t >> lane) & 1u) dst[into + __popc(t & low)] = slot;
    from += __popc(f);
    into += __popc(t);
  }
  cluster_sync();  // the lists of all slices are written; and no CTA leaves while a peer reads its shared memory
  if (scores_out == nullptr && positions_out == nullptr) return;
  // the moves, for the weights themselves: every slot read here is behind the budget, every slot written in front
  const int moves = __ldcg(P.n_moves + list);
  const int stride = static_cast<int>(n_cta) * kEvThreads;
  for (int j0 = static_cast<int>(rank) * kEvThreads + tid; j0 < moves; j0 += 4 * stride) {
    int s[4], d[4], pos[4];
    float w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (j0 + k * stride < moves) s[k] = __ldcg(src + j0 + k * stride), d[k] = __ldcg(dst + j0 + k * stride);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (j0 + k * stride >= moves) continue;
      if (scores_out != nullptr) w[k] = __ldcg(scores + s[k]);
      if (positions_out != nullptr) pos[k] = __ldcg(positions + s[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (j0 + k * stride >= moves) continue;
      if (scores_out != nullptr) scores_out[d[k]] = w[k];
      if (positions_out != nullptr) positions_out[d[k]] = pos[k];
    }
  }
  if (scores_out == nullptr || copy_scores) return;
  cluster_sync();  // in place: behind the budget all has been read
  for (int i = max(m, at) + tid; i < at + mine; i += kEvThreads) scores_out[i] = 0.f;
}

// ---- move_rows -----------------------------------------------------------------------------------
constexpr int kMoveThreads = 256;
constexpr int kMovePools = 32;
constexpr int kMoveMost = 256;  // moves of a block

struct MoveParams {
  unsigned char* pool[kMovePools];
  unsigned char* param[kMovePools];
  long long n_pages, s_page, s_kv, s_slot, s_head, p_page, p_kv, p_slot, p_head;
  const int *table, *src, *dst, *n_moves;
  int* status;
  long long table_stride, move_stride;
  int B, G, heads, page_size, units, words, per_block;  // units: 16-byte pieces of a row; words: 4-byte pieces of its params
  FastDiv by_page, by_heads, by_units, by_words;
};

// Where the row of a position begins in an array of the given strides, or -1.
struct Place {
  int page, slot;
};
__device__ __forceinline__ Place place_of(const MoveParams& P, int b, int pos) {
  Place p = {-1, 0};
  if (pos < 0) return p;
  const int pi = pos / P.by_page;
  p.page = static_cast<int>(page_of(P.table, P.table_stride, P.n_pages, b, pi));
  p.slot = pos - pi * P.page_size;
  return p;
}

// A block carries out up to per_block moves of one list in one pool: it looks up where their rows lie, then copies
// them in pieces of 16 bytes, four in flight to a thread, and their params in words.
__global__ void __launch_bounds__(kMoveThreads) move_rows_kernel(const __grid_constant__ MoveParams P) {
  __shared__ longlong2 row[kMoveMost], word[kMoveMost];  // offsets of source and destination; source -1: not to be moved
  const int b = blockIdx.y / P.G, g = blockIdx.y - b * P.G;
  const long long j0 = static_cast<long long>(blockIdx.x) * P.per_block;
  // (compared in 64 bits: a count near -2^31 less j0 would come out positive in 32, and row[] would be overrun)
  const long long left = min(static_cast<long long>(P.n_moves[blockIdx.y]), P.move_stride) - j0;
  if (left <= 0) return;
  const int n = static_cast<int>(min(left, static_cast<long long>(P.per_block)));
  const long long first = static_cast<long long>(blockIdx.y) * P.move_stride + j0;
  const int group = P.G > 1 ? g : 0;
  for (int j = threadIdx.x; j < n; j += kMoveThreads) {
    const Place from = place_of(P, b, P.src[first + j]), into = place_of(P, b, P.dst[first + j]);
    if (from.page < 0 || into.page < 0) {
      row[j] = word[j] = make_longlong2(-1, -1);
      if (P.status != nullptr) atomicOr(P.status + b, SPECATTN_ROW_BAD_INDEX);
      continue;
    }
    row[j] = make_longlong2(from.page * P.s_page + from.slot * P.s_slot + group * P.s_head, into.page * P.s_page + into.slot * P.s_slot + group * P.s_head);
    word[j] = make_longlong2(from.page * P.p_page + from.slot * P.p_slot + group * P.p_head, into.page * P.p_page + into.slot * P.p_slot + group * P.p_head);
  }
  __syncthreads();
  const int heads = P.G > 1 ? 1 : P.heads;  // of a group
  const FastDiv by_heads = P.by_heads;      // (by 1 where that is so)
  constexpr int kAhead = 4;
  {
    unsigned char* const pool = P.pool[blockIdx.z];
    const int total = n * 2 * heads * P.units;
    for (int x0 = threadIdx.x; x0 < total; x0 += kMoveThreads * kAhead) {
      uint4 v[kAhead];
      unsigned char* into[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int x = x0 + k * kMoveThreads;
        into[k] = nullptr;
        if (x >= total) continue;
        const int rest = x / P.by_units, up = rest / by_heads, h = rest - up * heads;
        const longlong2 at = row[up >> 1];
        if (at.x < 0) continue;
        const long long same = (up & 1 ? P.s_kv : 0) + h * P.s_head + (x - rest * P.units) * 16;
        into[k] = pool + at.y + same;
        v[k] = __ldcs(reinterpret_cast<const uint4*>(pool + at.x + same));
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (into[k] != nullptr) __stcs(reinterpret_cast<uint4*>(into[k]), v[k]);
    }
  }
  if (P.words == 0) return;
  unsigned char* const param = P.param[blockIdx.z];
  const int total = n * 2 * heads * P.words;
  for (int x0 = threadIdx.x; x0 < total; x0 += kMoveThreads * kAhead) {
    uint32_t v[kAhead];
    unsigned char* into[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int x = x0 + k * kMoveThreads;
      into[k] = nullptr;
      if (x >= total) continue;
      const int rest = x / P.by_words, up = rest / by_heads, h = rest - up * heads;
      const longlong2 at = word[up >> 1];
      if (at.x < 0) continue;
      const long long same = (up & 1 ? P.p_kv : 0) + h * P.p_head + (x - rest * P.words) * 4;
      into[k] = param + at.y + same;
      v[k] = *reinterpret_cast<const uint32_t*>(param + at.x + same);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (into[k] != nullptr) *reinterpret_cast<uint32_t*>(into[k]) = v[k];
  }
}

int clear_status(int32_t* status, size_t n, cudaStream_t stream) {
  if (status == nullptr || n == 0) return SPECATTN_OK;
  if (cudaMemsetAsync(status, 0, n * sizeof(int32_t), stream) == cudaSuccess) return SPECATTN_OK;
  cudaGetLastError();
  return SPECATTN_ERR_CUDA;
}

int launched() {
  if (cudaGetLastError() != cudaSuccess) return SPECATTN_ERR_CUDA;
  g_launch_count.fetch_add(1, std::memory_order_relaxed);
  return SPECATTN_OK;
}

}  // namespace
}  // namespace specattn

extern "C" int specattn_accumulate(const specattn_accumulate_args* args, void* cuda_stream) {
  using namespace specattn;
  NvtxRange nvtx_range("specattn_accumulate");
  if (args == nullptr) return SPECATTN_ERR_NULL;
  if (args->struct_size != sizeof(specattn_accumulate_args)) return SPECATTN_ERR_STRUCT_SIZE;
  const specattn_accumulate_args& A = *args;
  if (A.n_layers < 1 || A.n_layers > SPECATTN_MAX_DRAFT_LAYERS || A.batch < 0 || A.batch > 65535 || A.gamma < 1 || A.n_groups < 1 ||
      A.n_draft_heads < 1 || A.n_draft_heads > SPECATTN_MAX_DRAFT_HEADS || A.L_stride < 1 || A.L_stride > SPECATTN_MAX_KV_LEN ||
      A.score_stride < 1)
    return SPECATTN_ERR_RANGE;
  if (!(A.decay >= 0.) || isinf(A.decay)) return SPECATTN_ERR_RANGE;
  if (A.gamma > SPECATTN_MAX_ROWS_PER_LIST || static_cast<long long>(A.n_draft_heads) * A.gamma > SPECATTN_MAX_DRAFT_HEADS * SPECATTN_MAX_ROWS_PER_LIST)
    return SPECATTN_ERR_UNSUPPORTED;
  if (A.L_stride % 4 != 0) return SPECATTN_ERR_ALIGN;
  if (A.batch == 0) return SPECATTN_OK;
  if (!A.draft_probs || !A.kv_len || !A.scores_out) return SPECATTN_ERR_NULL;
  const bool grouped = A.head_group != nullptr && A.n_groups > 1;
  if (grouped && (A.n_groups > SPECATTN_MAX_DRAFT_HEADS || static_cast<long long>(A.batch) * A.n_groups > 65535)) return SPECATTN_ERR_UNSUPPORTED;
  AccParams P;
  memset(&P, 0, sizeof(P));
  bool any = false;
  for (int u = 0; u < A.n_layers; ++u) {
    P.probs[u] = A.draft_probs[u];
    any = any || P.probs[u] != nullptr;
    if (reinterpret_cast<uintptr_t>(P.probs[u]) % 16 != 0) return SPECATTN_ERR_ALIGN;
  }
  if (A.head_group != nullptr)
    for (int h = 0; h < A.n_draft_heads; ++h)
      if (A.head_group[h] < 0 || A.head_group[h] >= A.n_groups) return SPECATTN_ERR_RANGE;
  if (grouped) {
    int at = 0;
    for (int g = 0; g < A.n_groups; ++g) {
      P.first[g] = static_cast<unsigned short>(at);
      for (int h = 0; h < A.n_draft_heads; ++h)
        if (A.head_group[h] == g) P.head[at++] = static_cast<unsigned char>(h);
    }
    P.first[A.n_groups] = static_cast<unsigned short>(at);
  }
  P.kv_len = A.kv_len;
  P.in = A.scores_in;
  P.out = A.scores_out;
  P.row_status = A.row_status;
  P.L_stride = A.L_stride;
  P.score_stride = A.score_stride;
  P.decay = A.decay;
  P.B = A.batch;
  P.H = A.n_draft_heads;
  P.gamma = A.gamma;
  P.G = A.n_groups;
  P.grouped = grouped ? 1 : 0;
  const int sms = device_sm_count();
  if (sms <= 0) return SPECATTN_ERR_CUDA;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const int rc = clear_status(A.row_status, static_cast<size_t>(A.n_layers) * A.batch * A.n_groups, stream);
  if (rc != SPECATTN_OK || !any) return rc;
  // rows are dealt to more threads while the positions alone do not make 512 of them for every SM
  const long long width = A.L_stride < A.score_stride ? A.L_stride : A.score_stride;
  const long long quads = (width + 3) / 4, lists = static_cast<long long>(A.batch) * (grouped ? A.n_groups : 1);
  const long long threads = quads * lists * A.n_layers, rows = static_cast<long long>(A.n_draft_heads) * A.gamma / (grouped ? A.n_groups : 1);
  int slices = 1;
  while (slices < 8 && threads * slices < 512ll * sms && rows > 4 * slices) slices *= 2;
  const dim3 grid(static_cast<unsigned>((quads * slices + kAccThreads - 1) / kAccThreads), static_cast<unsigned>(lists), A.n_layers);
  switch (slices) {
    case 1: accumulate_kernel<1><<<grid, kAccThreads, 0, stream>>>(P); break;
    case 2: accumulate_kernel<2><<<grid, kAccThreads, 0, stream>>>(P); break;
    case 4: accumulate_kernel<4><<<grid, kAccThreads, 0, stream>>>(P); break;
    default: accumulate_kernel<8><<<grid, kAccThreads, 0, stream>>>(P); break;
  }
  return launched();
}

extern "C" int specattn_evict(const specattn_evict_args* args, void* cuda_stream) {
  using namespace specattn;
  NvtxRange nvtx_range("specattn_evict");
  if (args == nullptr) return SPECATTN_ERR_NULL;
  if (args->struct_size != sizeof(specattn_evict_args)) return SPECATTN_ERR_STRUCT_SIZE;
  const specattn_evict_args& A = *args;
  if (A.n_layers < 1 || A.batch < 0 || A.n_groups < 1 || A.L < 1 || A.L > SPECATTN_MAX_KV_LEN || A.budget < 1 || A.n_sink < 0 ||
      A.n_recent < 0 || static_cast<long long>(A.n_sink) + A.n_recent > A.budget || A.reserved != 0)
    return SPECATTN_ERR_RANGE;
  const long long room = A.L - A.budget < A.budget ? A.L - A.budget : A.budget;
  if (A.move_stride < (room > 0 ? room : 0)) return SPECATTN_ERR_RANGE;
  const long long lists = static_cast<long long>(A.n_layers) * A.batch * A.n_groups;
  if (lists > (1ll << 24)) return SPECATTN_ERR_UNSUPPORTED;
  if (A.batch == 0) return SPECATTN_OK;
  if (!A.scores || !A.kv_len || !A.n_moves || !A.new_len || (room > 0 && (!A.src || !A.dst))) return SPECATTN_ERR_NULL;
  if (A.positions_out != nullptr && A.positions == nullptr) return SPECATTN_ERR_NULL;
  if (A.new_len == A.kv_len || A.new_len == A.seq_len) return SPECATTN_ERR_RANGE;
  EvictParams P;
  P.scores = A.scores;
  P.kv_len = A.kv_len;
  P.positions = A.positions;
  P.seq_len = A.seq_len;
  P.src = A.src;
  P.dst = A.dst;
  P.n_moves = A.n_moves;
  P.new_len = A.new_len;
  P.scores_out = A.scores_out;
  P.positions_out = A.positions_out;
  P.L = A.L;
  P.move_stride = A.move_stride;
  P.budget = A.budget;
  P.n_sink = A.n_sink;
  P.n_recent = A.n_recent;
  P.B = A.batch;
  P.G = A.n_groups;
  const int sms = device_sm_count();
  if (sms <= 0) return SPECATTN_ERR_CUDA;
  // CTAs to a list: enough for 16384 slots or fewer to each (40 lists of 32768, one or two CTAs to an SM are 26 to 29 us; 300
  // of 20000 whole 95, halved 74); more while every one has an SM to itself and 1024 slots (8 lists of 32768 with 2 / 4 / 8:
  // 27.6 / 18.8 / 14.8 us, one of 4096 with 1 / 2 / 4 / 8: 12.6 / 11.1 / 10.3 / 10.6)
  int ctas = 1;
  const auto slots = [&] { return (A.L + ctas - 1) / ctas; };
  while (ctas < kEvMaxCluster && (slots() > 16384 || (lists * ctas * 2 <= sms && slots() >= 2048))) ctas *= 2;
  P.slice = static_cast<int>(((A.L + ctas - 1) / ctas + 3) / 4 * 4);
  P.wide = A.L % 4 == 0 && ((reinterpret_cast<uintptr_t>(A.scores) | reinterpret_cast<uintptr_t>(A.positions) |
                             reinterpret_cast<uintptr_t>(A.scores_out) | reinterpret_cast<uintptr_t>(A.positions_out)) % 16 == 0);
  const size_t smem = static_cast<size_t>(P.slice) * sizeof(uint32_t);
  // 1024 threads for many slots on an SM of their own (74 lists of 32768 by halves 26.6 against 29.1 us); of 512 two CTAs fit, and
  // fewer slots do not fill more (8 lists of 32768 by eighths 14.8 against 15.3, 224 of 2667 15.7 against 23.9)
  const bool many = slots() < 8192 || lists * ctas > sms;
  const auto kernel = many ? evict_kernel<512> : evict_kernel<1024>;
  static std::atomic<unsigned long long> prepared[2];  // a bit per device
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return SPECATTN_ERR_CUDA;
  }
  if (!((prepared[many].load(std::memory_order_acquire) >> dev) & 1ull)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kEvMaxSlice * 4) != cudaSuccess) {
      cudaGetLastError();
      return SPECATTN_ERR_CUDA;
    }
    prepared[many].fetch_or(1ull << dev, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(static_cast<unsigned>(lists * ctas));
  cfg.blockDim = dim3(many ? 512 : 1024);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(cuda_stream);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, P) != cudaSuccess) {
    cudaGetLastError();
    return SPECATTN_ERR_CUDA;
  }
  g_launch_count.fetch_add(1, std::memory_order_relaxed);
  return SPECATTN_OK;
}

extern "C" int specattn_move_rows(const specattn_move_args* args, void* cuda_stream) {
  using namespace specattn;
  NvtxRange nvtx_range("specattn_move_rows");
  if (args == nullptr) return SPECATTN_ERR_NULL;
  if (args->struct_size != sizeof(specattn_move_args)) return SPECATTN_ERR_STRUCT_SIZE;
  const specattn_move_args& A = *args;
  if (A.stride_page < 0 || A.stride_kv < 0 || A.stride_slot < 0 || A.stride_head < 0 || A.pstride_page < 0 || A.pstride_kv < 0 ||
      A.pstride_slot < 0 || A.pstride_head < 0 || A.n_pools < 0 || A.batch < 0 || A.n_kv_heads < 1 || A.page_size < 1 || A.n_pages < 1 || A.n_pages > INT32_MAX ||
      (A.n_groups != 1 && A.n_groups != A.n_kv_heads) || A.block_table_stride < 0 || A.move_stride < 0 || A.row_bytes < 16 ||
      A.row_bytes > 4096 || A.param_bytes < 0 || A.param_bytes > 256)
    return SPECATTN_ERR_RANGE;
  if (static_cast<long long>(A.batch) * A.n_groups > 65535 || A.n_kv_heads > 1024) return SPECATTN_ERR_UNSUPPORTED;
  if ((A.param_bytes != 0) != (A.params != nullptr)) return SPECATTN_ERR_NULL;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (A.batch == 0) return SPECATTN_OK;
  if (!A.n_moves || (A.n_pools > 0 && !A.pools) || (A.move_stride > 0 && (!A.src || !A.dst))) return SPECATTN_ERR_NULL;
  if (A.row_bytes % 16 || A.stride_page % 16 || A.stride_kv % 16 || A.stride_slot % 16 || A.stride_head % 16 || A.param_bytes % 4 ||
      A.pstride_page % 4 || A.pstride_kv % 4 || A.pstride_slot % 4 || A.pstride_head % 4)
    return SPECATTN_ERR_ALIGN;
  for (int i = 0; i < A.n_pools; ++i) {
    if (!A.pools[i] || (A.params && !A.params[i])) return SPECATTN_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(A.pools[i]) % 16 != 0 || (A.params && reinterpret_cast<uintptr_t>(A.params[i]) % 4 != 0))
      return SPECATTN_ERR_ALIGN;
  }
  const int rc = clear_status(A.status, static_cast<size_t>(A.batch), stream);
  if (rc != SPECATTN_OK || A.move_stride == 0) return rc;
  MoveParams P;
  memset(&P, 0, sizeof(P));
  P.n_pages = A.n_pages;
  P.s_page = A.stride_page;
  P.s_kv = A.stride_kv;
  P.s_slot = A.stride_slot;
  P.s_head = A.stride_head;
  P.p_page = A.pstride_page;
  P.p_kv = A.pstride_kv;
  P.p_slot = A.pstride_slot;
  P.p_head = A.pstride_head;
  P.table = A.block_table;
  P.table_stride = A.block_table_stride;
  P.src = A.src;
  P.dst = A.dst;
  P.n_moves = A.n_moves;
  P.status = A.status;
  P.move_stride = A.move_stride;
  P.B = A.batch;
  P.G = A.n_groups;
  P.heads = A.n_kv_heads;
  P.page_size = A.page_size;
  P.units = static_cast<int>(A.row_bytes / 16);
  P.words = static_cast<int>(A.param_bytes / 4);
  P.by_page = fast_div(A.page_size);
  P.by_heads = fast_div(A.n_groups > 1 ? 1 : A.n_kv_heads);
  P.by_units = fast_div(P.units);
  P.by_words = fast_div(P.words > 0 ? P.words : 1);
  // about 64 KB to a block: long enough to hide the lookups, short enough to spread a few moves
  const long long bytes = 2 * A.row_bytes * (A.n_groups > 1 ? 1 : A.n_kv_heads);
  long long per = 65536 / bytes;
  if (per < 1) per = 1;
  if (per > kMoveMost) per = kMoveMost;
  // (few moves are spread over the SMs: latency is all there is to them)
  const int sms = device_sm_count();
  if (sms <= 0) return SPECATTN_ERR_CUDA;
  while (per > 4 && (A.move_stride + per - 1) / per * A.batch * A.n_groups * A.n_pools < 2ll * sms) per /= 2;
  P.per_block = static_cast<int>(per);
  const long long blocks = (A.move_stride + per - 1) / per;
  if (blocks > INT32_MAX) return SPECATTN_ERR_UNSUPPORTED;
  for (int i0 = 0; i0 < A.n_pools; i0 += kMovePools) {
    const int n = A.n_pools - i0 < kMovePools ? A.n_pools - i0 : kMovePools;
    for (int i = 0; i < n; ++i) {
      P.pool[i] = static_cast<unsigned char*>(A.pools[i0 + i]);
      P.param[i] = A.params ? static_cast<unsigned char*>(A.params[i0 + i]) : nullptr;
    }
    move_rows_kernel<<<dim3(static_cast<unsigned>(blocks), A.batch * A.n_groups, n), kMoveThreads, 0, stream>>>(P);
    const int lc = launched();
    if (lc != SPECATTN_OK) return lc;
  }
  return SPECATTN_OK;
}
