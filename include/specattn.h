/* specattn.h -- C ABI of the SpecAttn verification hot path for NVIDIA B200 (sm_100a).
 *
 * The library implements, as hand-written CUDA kernels, the per-step work that the SpecAttn
 * verifier performs for each of its layers:
 *
 *   select:  sum the mapped draft layer's attention probabilities over draft heads and the
 *            gamma speculated queries, find the exact top-p nucleus of context positions
 *            without sorting (a radix threshold search over the binary32 bit pattern with
 *            per-bin counts and masses) and emit the kept positions as ascending index lists.
 *   verify:  grouped-query sparse decode attention of the gamma+1 verification queries over
 *            only the listed rows of a paged bf16 K/V cache, returning outputs and LSE.
 *
 * Conventions common to every entry point
 *   - Pointers are DEVICE pointers unless the comment says HOST.  The caller owns every
 *     buffer; the library never allocates or frees device memory and never synchronises.
 *     Work is enqueued on the CUDA stream passed as `cuda_stream` (a cudaStream_t cast to
 *     void*; NULL = the legacy default stream) and is complete when that stream reaches it.
 *   - Return value: SPECATTN_OK (0) = enqueued; a negative SPECATTN_ERR_* = argument error
 *     detected on the host, nothing was launched.  Data-dependent problems are reported per
 *     list / per sequence in device status words as SPECATTN_ROW_* bit flags; the device
 *     code never traps.
 *   - `struct_size` must be sizeof() of the struct the caller was compiled against.
 *   - Strides are in ELEMENTS of the array they index.
 *   - Tracing: specattn_select_topp, specattn_sparse_verify, specattn_verify_plan(_many) and
 *     specattn_verify_step_host each open an NVTX range of their own name around their host-side
 *     work (visible in a profiler's timeline; a null-pointer test when no tool is attached).
 */
#ifndef SPECATTN_H_
#define SPECATTN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- host-side return codes ------------------------------------------------------------ */
#define SPECATTN_OK 0
#define SPECATTN_ERR_NULL (-1)        /* a required pointer is NULL */
#define SPECATTN_ERR_STRUCT_SIZE (-2) /* struct_size does not match this library */
#define SPECATTN_ERR_RANGE (-3)       /* a scalar is outside its documented range */
#define SPECATTN_ERR_ALIGN (-4)       /* a pointer or stride breaks the 16-byte rules */
#define SPECATTN_ERR_WORKSPACE (-5)   /* workspace missing or smaller than *_workspace_bytes() */
#define SPECATTN_ERR_UNSUPPORTED (-6) /* shape outside what the kernels are built for */
#define SPECATTN_ERR_CUDA (-7)        /* the CUDA runtime refused the launch */
#define SPECATTN_ERR_STATIC_SCRATCH (-8) /* shape needs more scratch than the built-in buffer has */

/* ---- device-side per-list / per-sequence status flags ---------------------------------- */
#define SPECATTN_ROW_OK 0
#define SPECATTN_ROW_INVALID_PROB 1 /* a contributing probability was negative, NaN or Inf (or the
                                       binary32 sum of a position overflowed) */
#define SPECATTN_ROW_OVERFLOW 2     /* the list has more entries than idx_stride; truncated */
#define SPECATTN_ROW_BAD_INDEX 4    /* verify met a position or page id out of range */
#define SPECATTN_ROW_TIMEOUT 8      /* a bounded device-side wait ran out; outputs invalid */
#define SPECATTN_ROW_INVALID_VALUE 16 /* a K/V row held NaN or an infinity, or spans more than binary32 */

/* ---- limits ---------------------------------------------------------------------------- */
#define SPECATTN_MAX_DRAFT_LAYERS 64
#define SPECATTN_MAX_DRAFT_HEADS 256
#define SPECATTN_MAX_ROWS_PER_LIST 1024  /* contributing (head, query) rows per list */
#define SPECATTN_MAX_KV_LEN 196608       /* positions per sequence for select         */
#define SPECATTN_MAX_VERIFY_UNITS 2048   /* batch * n_kv_heads for verify */
#define SPECATTN_MAX_QUERY_ROWS 64       /* n_q * (n_q_heads / n_kv_heads) for verify */

/* ========================================================================================
 * specattn_select_topp -- token selection.
 *
 * Paper: Sec. 3.4 ("Sorting-Free Top-p Nucleus Selection"), Alg. 2, and the top-p objective
 * of App. A Eq. 7; the per-layer use is Alg. 1, block "Sparse Attention Mask Creation".
 *
 * For every draft layer u that some target layer maps to (layer_map[j] == u), every sequence
 * b and every group g:
 *   a_bar[i] = +0 + sum over heads h feeding g (ascending) of sum over s < gamma (ascending)
 *              of draft_probs[u][b, h, s, i],   i < kv_len[b]        (binary32 adds, this order)
 *   total    = sum_i a_bar[i];  target = (double) p * total            (Alg. 2: p * sum a)
 *   theta    = the largest row value v whose mass {a_bar >= v} reaches target -- the fixed
 *              point of Alg. 2's bisection, identical to the sorted-prefix nucleus of Eq. 7
 *   list     = ascending { i : a_bar[i] >= theta }  (ties at theta all kept)
 *   p >= 1 keeps every position; an all-zero row keeps every position.
 * Draft layers no target layer maps to are skipped and their outputs left untouched.
 *
 * Outputs per (u, b, g), all indexed [n_draft_layers, batch, n_groups]:
 *   idx     int32 [.., idx_stride]: the list, first min(count, idx_stride) entries
 *   counts  int32: the true list length (also when it exceeds idx_stride)
 *   row_status int32: SPECATTN_ROW_* flags.  INVALID_PROB => count 0, list unspecified.
 *   diag    optional double [.., 4] = {total, target, mass strictly above theta,
 *           mass of the kept set}; NULL to skip.
 *
 * Variants of Alg. 2 (both off by default; results differ from the exact nucleus by design):
 *   per_step = 1: Alg. 2 as printed -- every speculated query s gets its own row
 *       a_s[i] = +0 + sum over heads h feeding g (ascending) of draft_probs[u][b, h, s, i], its
 *       own threshold, and the list is the ascending union of the gamma sets.
 *   bisect_iters = n in [1, 64]: the threshold of a row is the LAST midpoint of n bisection
 *       steps (theta_high = max of the row, theta_low = 0, theta_mid = (high + low) / 2 in
 *       binary32; mass of {a >= theta_mid} < target lowers theta_high, otherwise raises
 *       theta_low) -- the paper's implementation uses n = 10.  The set {a >= theta_mid} may fall
 *       short of the target mass or exceed the smallest set.  p >= 1 and all-zero rows still
 *       keep every position.  diag then describes the exact threshold of the last row searched.
 *
 *   chunk = c in {4, 8, 16, 32, 64} (0 or 1 = off): selection at chunk granularity (Sec. 4 sets
 *       the chunk size to 16; how a chunk is scored is not stated -- here: its score is
 *       +0 + a[c j] + a[c j + 1] + ... in binary32, ascending, the last chunk cut at kv_len).  The
 *       nucleus (either variant above applies) is taken over the row of chunk scores and a kept
 *       chunk keeps all its positions; counts / idx_stride stay in positions.
 *
 * Requirements: 1 <= n_draft_layers <= 64; n_draft_heads <= 256; gamma >= 1; L_stride a
 * multiple of 4 and <= SPECATTN_MAX_KV_LEN; every draft_probs[u] 16-byte aligned;
 * 0 <= kv_len[b] <= L_stride (larger values are clamped); 0 < p (NaN rejected);
 * n_groups >= 1; head_group (HOST, may be NULL = every head feeds every group) values in
 * [0, n_groups).
 *
 * workspace (optional, device, 16-byte aligned, specattn_select_workspace_bytes() bytes; no
 * counterpart in the paper): without it each list is aggregated and searched inside the shared
 * memory of one thread-block cluster (at most 16 CTAs per list, one launch).  With it, and for
 * the default selection (no variant) over rows of >= 2048 positions when the lists are so few
 * that one cluster each would leave SMs idle (lists x CTAs per cluster, at most 8, < 148), the call runs two
 * launches: every list's rows are summed by CTAs of 512 positions each -- in the same order,
 * so a[] has the same bits -- into the workspace, and the search then reads a[] from there; the
 * lists are the same, the GPU is filled whatever the number of lists.  The workspace holds no
 * state between calls; two calls that may overlap on the GPU need separate workspaces.
 *
 * form: which of the two the call takes when both apply (a workspace is given, default selection,
 * multi-row lists of >= 2048 positions).  SPECATTN_SELECT_FORM_AUTO decides by what the host
 * can see (the number of lists).  What it cannot see is kv_len: in a ragged batch one cluster per
 * list means the longest list sets the time while most of the GPU is done, and the two-launch
 * form, whose first launch spends CTAs in proportion to each list's length, is the better one --
 * a caller that knows its batch is ragged says SPECATTN_SELECT_FORM_TWO_LAUNCH
 * (specattn_select_workspace_bytes then answers for that form).  SPECATTN_SELECT_FORM_CLUSTER
 * keeps one launch.  The lists are the same bits in every form.
 * ======================================================================================== */
#define SPECATTN_SELECT_FORM_AUTO 0
#define SPECATTN_SELECT_FORM_CLUSTER 1
#define SPECATTN_SELECT_FORM_TWO_LAUNCH 2

typedef struct specattn_select_args {
  uint32_t struct_size;
  int32_t n_draft_layers;
  int32_t n_target_layers;
  int32_t batch;
  int32_t n_draft_heads;
  int32_t gamma;
  int32_t n_groups;
  int64_t L_stride;
  const float* const* draft_probs; /* HOST array [n_draft_layers] of device pointers to
                                      binary32 [batch, n_draft_heads, gamma, L_stride];
                                      entries of unmapped layers may be NULL */
  const int32_t* kv_len;           /* [batch] */
  const int32_t* layer_map;        /* HOST [n_target_layers], values in [-1, n_draft_layers);
                                      -1 marks a dense target layer */
  const int32_t* head_group;       /* HOST [n_draft_heads] or NULL */
  float p;
  int32_t* idx;
  int64_t idx_stride;
  int32_t* counts;
  int32_t* row_status;
  double* diag;
  int32_t per_step;     /* 0 | 1 */
  int32_t bisect_iters; /* 0 = exact threshold, else 1..64 */
  int32_t chunk;        /* 0 | 1 = per position, else 4, 8, 16, 32 or 64 */
  int32_t form;         /* SPECATTN_SELECT_FORM_*: 0 = the library picks */
  void* workspace;          /* device, or NULL */
  uint64_t workspace_bytes; /* size of *workspace */
} specattn_select_args;

int specattn_select_topp(const specattn_select_args* args, void* cuda_stream);

/* Bytes of workspace that let specattn_select_topp(args) take its two-launch form (0 when the
 * call would not use one: a variant, single-row lists, rows shorter than 2048 positions, enough
 * lists to fill the GPU with one cluster each, or invalid arguments).  Reads only the scalar fields and layer_map of args. */
size_t specattn_select_workspace_bytes(const specattn_select_args* args);

/* ========================================================================================
 * specattn_sparse_verify -- sparse attention of one target layer.
 *
 * Paper: Eq. 1 restricted to the selected index set I of Eq. 2-3 (softmax normalised over I;
 * the un-normalised form of Eq. 2 is out * exp(lse - lse_dense)); Sec. 3.5; Alg. 1, block
 * "Verification with Sparse Attention" (one list per layer shared by all gamma+1 queries).
 *
 * For sequence b, query t < n_q and query head h (kv head hk = h / (n_q_heads/n_kv_heads),
 * list g = 0 if n_groups == 1 else hk):
 *   s_i = sm_scale * q[b,t,h,:] . K[i, hk, :]  for i in the list;  m = max s_i
 *   out[b,t,h,:] = sum_i exp(s_i - m) V[i, hk, :] / sum_i exp(s_i - m)
 *   lse[b,t,h]   = m + ln sum_i exp(s_i - m)          (natural log)
 * An empty list gives out = 0, lse = -inf.  Position i of sequence b lives in page
 * block_table[b * block_table_stride + i / page_size] at slot i % page_size; with
 * block_table == NULL the cache is contiguous and that page is
 * b * block_table_stride + i / page_size (block_table_stride = pages per sequence).
 * Element (page, kv, slot, head, e) of kv_pages is at
 *   page*stride_page + kv*stride_kv + slot*stride_slot + head*stride_head + e,
 * kv = 0 for keys and 1 for values.
 *
 * idx / counts point at the lists of ONE draft layer: idx [batch, n_groups, idx_stride],
 * counts [batch, n_groups] (entries beyond idx_stride are ignored).  dense != 0 attends every
 * position below kv_len[b] and reads neither idx nor counts (both may be NULL).
 *
 * tail_len > 0 adds the tokens being verified themselves (Alg. 1: the gamma+1 tokens go through
 * the verifier in one pass): their K/V rows must already be in the cache at positions
 * kv_len[b] + j, j < tail_len, and query t attends, after its list, the rows with
 * j <= t + (tail_len - n_q) -- with tail_len == n_q token t sees tokens 0..t.  kv_len stays the
 * context length without them.
 *
 * Requirements: head_dim == 128; n_q * (n_q_heads / n_kv_heads) <= 64; batch * n_kv_heads
 * <= 2048; q, kv_pages 16-byte aligned and all four strides multiples of 8; out 16-byte
 * aligned.  status (int32 [batch], optional) receives SPECATTN_ROW_BAD_INDEX when a listed
 * position is outside [0, kv_len[b]) or a page id outside [0, n_pages) (such entries are
 * read from position 0 / page 0 instead; n_pages == 0 disables the page check).
 *
 * workspace: at least specattn_verify_workspace_bytes() bytes, 256-byte aligned, prepared
 * once with specattn_verify_workspace_init() and then reusable by consecutive calls on the
 * same stream; two calls that may overlap on the GPU need separate workspaces.  (Up to 24 query rows per KV head
 * and more (sequence, KV head) pairs than half of the SMs: two CTAs share an SM and need more workspace than
 * one would.  A call with less, down to what one CTA per SM needs, runs with one; its results are the same within the
 * tolerance of the operation, not bit for bit.)
 * ======================================================================================== */
/* flags for specattn_verify_args.flags
 *
 * SPECATTN_VERIFY_LISTS_STABLE: the caller promises that idx, counts, kv_len, block_table and
 * the listed rows of kv_pages were produced at least two launches earlier in the stream, and
 * that the launch right before this call is either another specattn_sparse_verify call or a
 * kernel that does not signal programmatic launch completion early.  (True for every layer
 * after the first of a step: the lists come from specattn_select_topp and the context's K/V
 * rows are old.)  The verify kernel is always launched with programmatic stream
 * serialization, i.e. it may begin while the preceding kernel is still running.  Without this
 * flag it waits for that kernel to finish before reading anything, and lets its own successor
 * start only after that wait; with it, it starts fetching K/V rows at once and waits only
 * before reading q and before writing out, lse, status or the workspace.
 *
 * SPECATTN_VERIFY_ENGINE_MMA_SYNC / SPECATTN_VERIFY_ENGINE_TCGEN05: force one of the two
 * implementations of the same operation (warp-level mma.sync with register accumulators, or
 * tcgen05.mma with accumulators in tensor memory).  With neither bit the library picks by
 * what the host can see: tcgen05 for dense calls over caches of at least 8192 positions per
 * sequence (block_table_stride * page_size) that either have more than 32 query rows per KV head
 * (n_q * n_q_heads / n_kv_heads) or can be read page-wise (page_size a multiple of 16, n_pages
 * given), mma.sync otherwise -- list lengths live on the device, so a
 * caller that knows its lists are long (thousands of positions per sequence) and has more than
 * 32 query rows should set SPECATTN_VERIFY_ENGINE_TCGEN05 itself.  Results agree within the
 * tolerance of the operation either way.  Setting both bits is SPECATTN_ERR_RANGE. */
#define SPECATTN_VERIFY_LISTS_STABLE 1u
#define SPECATTN_VERIFY_ENGINE_MMA_SYNC 2u
#define SPECATTN_VERIFY_ENGINE_TCGEN05 4u
/* SPECATTN_VERIFY_PAGE_LISTS: the caller promises that every list consists of whole aligned
 * 16-position chunks -- entries 16 a ... 16 a + 15 are 16 consecutive positions starting at a
 * multiple of 16, for every a; only the last chunk of a list may be shorter (cut at kv_len or at
 * idx_stride).  Lists written by specattn_select_topp with chunk = 16, 32 or 64 have this form
 * (Sec. 4: chunk size 16).  Where the cache's page size is a multiple of 16 and n_pages is given,
 * the kernel then reads K/V page-wise -- one list entry, one block-table entry and four tiled
 * bulk tensor copies (16 slots x 128 bytes each) per 16 tokens instead of 16 entries and 512
 * 16-byte copies -- and so does every dense call.  A list that breaks the promise gives wrong
 * results for its sequence (entries that are not multiples of 16 raise SPECATTN_ROW_BAD_INDEX),
 * never a fault.  Results are the same as without the flag. */
#define SPECATTN_VERIFY_PAGE_LISTS 8u
/* SPECATTN_VERIFY_INIT_WORKSPACE / SPECATTN_VERIFY_INIT_STATUS: the call itself clears, on the stream and
 * ahead of its kernel, the workspace's arrival counters that it uses (the workspace needs no
 * specattn_verify_workspace_init before this call; nor can another call rely on it afterwards
 * unless that call has at most this one's batch * n_kv_heads) / the status words.  One small kernel for
 * both, which the verify kernel overlaps: cheaper than two memsets in front of a call that allocates
 * its workspace anew. */
#define SPECATTN_VERIFY_INIT_WORKSPACE 16u
#define SPECATTN_VERIFY_INIT_STATUS 32u
/* TEST ONLY -- never set this in production.  Exercises the failure path of the kernels' bounded
 * device-side waits without faulting anything: one producer warp of CTA 0 withholds the
 * completion signal of its first tile, the waits on it give up after their poll limit (about
 * half a second each), the CTA raises SPECATTN_ROW_TIMEOUT in status[0] and the kernel returns
 * normally.  Outputs of that call are invalid and the workspace must be re-initialised with
 * specattn_verify_workspace_init before its next use. */
#define SPECATTN_VERIFY_TEST_LOSE_ARRIVAL 0x80000000u

typedef struct specattn_verify_args {
  uint32_t struct_size;
  int32_t batch;
  int32_t n_q;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t page_size;
  int32_t n_groups;
  int32_t dense;
  const void* q;        /* bf16 [batch, n_q, n_q_heads, head_dim] */
  const void* kv_pages; /* bf16 pool of this target layer */
  int64_t n_pages;
  int64_t stride_page, stride_kv, stride_slot, stride_head;
  const int32_t* block_table;
  int64_t block_table_stride;
  const int32_t* kv_len; /* [batch] */
  const int32_t* idx;
  int64_t idx_stride;
  const int32_t* counts;
  float sm_scale;        /* > 0, or 0 => 1/sqrt(head_dim); negative or NaN is rejected */
  float* out;            /* binary32 [batch, n_q, n_q_heads, head_dim] */
  float* lse;            /* binary32 [batch, n_q, n_q_heads] */
  int32_t* status;       /* [batch] or NULL */
  void* workspace;
  size_t workspace_bytes;
  uint32_t flags;        /* SPECATTN_VERIFY_* bits, 0 for none */
  int32_t tail_len;      /* in-flight tokens attended causally after the list, 0 <= tail_len <= 64 */
  const void* plan;      /* optional: a work partition made by specattn_verify_plan, or NULL */
} specattn_verify_args;

/* Bytes of workspace specattn_sparse_verify needs for these shapes on the current device
 * (0 on argument error).  Depends only on the scalar fields. */
size_t specattn_verify_workspace_bytes(const specattn_verify_args* args);

/* Zero the arrival counters at the head of a verify workspace (enqueued on the stream).
 * Call once after allocating it; the kernels leave the counters zero when they finish. */
int specattn_verify_workspace_init(void* workspace, size_t workspace_bytes, void* cuda_stream);

int specattn_sparse_verify(const specattn_verify_args* args, void* cuda_stream);

/* specattn_verify_plan -- the work partition of a verify launch, computed ahead of it.
 *
 * Not an operation of the paper: an engineering shortcut of this implementation.  How the kernel
 * deals its (sequence, kv head) lists to the SMs depends only on the list lengths (counts, or
 * kv_len for dense calls), tail_len, the shapes (n_q, idx_stride and the room of the block table among
 * them) and the GPU -- not on q, the K/V pool or the outputs.  Target layers that share a draft layer's lists therefore share the partition, and a
 * verify kernel that finds a matching plan in args->plan skips computing it (a few microseconds
 * of start-up per launch).  `plan` is a device buffer of specattn_verify_plan_bytes(args) bytes,
 * 16-byte aligned, written by a small kernel on the stream (after whatever produces counts /
 * kv_len, e.g. specattn_select_topp) and valid until those change.  A kernel given a plan that
 * does not fit its launch (other batch, heads, tail_len, dense flag, GPU, or a shape that is launched
 * in clusters of another size or with another number of CTAs) ignores it.  Only
 * the mma.sync engine reads plans.
 * A plan is for the workspace in its arguments: with args->workspace set and workspace_bytes below
 * specattn_verify_workspace_bytes(args) it fits calls with such a smaller workspace, otherwise those with
 * the full one and specattn_sparse_verify_static.
 * Ordering: a plan must be at least as new as the lists it describes -- call this after every
 * specattn_select_topp that rewrites counts -- and a verify call flagged
 * SPECATTN_VERIFY_LISTS_STABLE must not be the first launch after the plan kernel (that flag's
 * "two launches earlier" rule covers the plan like the lists): the plan kernel signals completion
 * only when it has finished, and the first verify call after it waits for that. */
size_t specattn_verify_plan_bytes(const specattn_verify_args* args);
int specattn_verify_plan(const specattn_verify_args* args, void* plan, size_t plan_bytes, void* cuda_stream);
/* The same for n launches at once (HOST arrays of n argument structs, plan buffers and their
 * sizes): one kernel launch per eight plans instead of one per plan -- a step whose target
 * layers share the lists of four draft layers needs four plans. */
int specattn_verify_plan_many(const specattn_verify_args* const* args, void* const* plans,
                              const size_t* plan_bytes, int32_t n, void* cuda_stream);

/* ========================================================================================
 * specattn_sparse_verify_static -- specattn_sparse_verify for callers that cannot allocate.
 *
 * (No counterpart in the paper: this entry point exists only for integration.)
 *
 * Some callers have no way to obtain the scratch buffer specattn_sparse_verify wants: code
 * running as a custom call inside another runtime's compiled graph is handed its input and
 * output buffers and nothing else; a serving engine may have reserved all device memory in
 * its own pool, so that a cudaMalloc from a plug-in fails or stalls the whole device; and
 * an allocation in the middle of a latency-critical decode loop synchronises the GPU.
 * For them this variant keeps the scratch inside the library: a file-scope
 * `static __device__` array (8 MiB) that every GPU loading the library holds from load until the
 * process exits.  The call allocates and frees nothing
 * (no cudaMalloc, cudaFree or allocating library routine).
 *
 * Same arguments, results and status codes as specattn_sparse_verify, except:
 *   - args->workspace and args->workspace_bytes are ignored;
 *   - a shape that needs more scratch than SPECATTN_STATIC_SCRATCH_BYTES with one CTA per SM is rejected with
 *     SPECATTN_ERR_STATIC_SCRATCH and nothing is launched.  The buffer covers up to 32 query rows per
 *     KV head (n_q * group <= 32) on GPUs with up to 160 SMs (there it also holds what two CTAs per SM
 *     need in batches of many sequences);
 *   - the first call on each device looks up the device address of the array (with that
 *     device current); make that first call outside any stream capture;
 *   - all calls on a device share the one array, which still holds what the previous call left
 *     there: the arrival counters are cleared on the stream at the start of every call, and
 *     two calls that may overlap on the GPU (different streams, or concurrent graph branches)
 *     race on it -- serialise them or use specattn_sparse_verify with separate workspaces;
 *   - the clearing is a memset in front of the launch, so a call flagged
 *     SPECATTN_VERIFY_LISTS_STABLE gains nothing here: the kernel cannot begin under its
 *     predecessor as it does after specattn_sparse_verify, it starts when the memset is done;
 *   - every argument check happens before the memset is enqueued: a negative return code means
 *     that nothing at all was enqueued.
 * ======================================================================================== */
#define SPECATTN_STATIC_SCRATCH_BYTES (6u << 20)

int specattn_sparse_verify_static(const specattn_verify_args* args, void* cuda_stream);

/* ========================================================================================
 * specattn_verify_step_host -- one whole verification step from HOST buffers.
 *
 * Alg. 1, blocks "Sparse Attention Mask Creation" and "Verification with Sparse Attention":
 * one select over the mapped draft layers, then one sparse verify per target layer, with the
 * step's inputs and results crossing PCIe inside the call.  It
 *   1. copies q_host[j] -> verify[j].q for every target layer and draft_probs_host[u] ->
 *      select.draft_probs[u] for every mapped draft layer, on a copy stream of its own,
 *   2. on the caller's stream runs specattn_select_topp for a draft layer as soon as its rows
 *      have landed (one launch per mapped draft layer) and then specattn_sparse_verify(verify[j])
 *      of the target layers mapped to it, while later draft layers are still being copied,
 *   3. copies verify[j].out / .lse -> out_host[j] / lse_host[j] on a second copy stream as each
 *      layer finishes,
 * and finally makes the caller's stream wait for both copy streams: work enqueued on that
 * stream afterwards sees the step complete.  The two copy streams and the events between the
 * lanes are created on the first call per device and kept; one call at a time enqueues per
 * device.  select.n_target_layers must equal n_target_layers.  Where verify[j].plan is set, the
 * call runs specattn_verify_plan into it before the first layer that points at it.
 * `select` and `verify[j]` are complete device-side argument structs (their device buffers,
 * including the staging buffers the copies land in, are the caller's); verify[j].idx/counts
 * must already point at the lists of layer_map[j] (or dense be set where layer_map[j] < 0).
 * Host buffers should be pinned for the copies to be asynchronous.  Nothing is synchronised:
 * the results are in the host buffers once the stream has drained.
 * ======================================================================================== */
typedef struct specattn_step_host_args {
  uint32_t struct_size;
  int32_t n_target_layers;
  const specattn_select_args* select;     /* HOST */
  const float* const* draft_probs_host;   /* HOST [n_draft_layers] of HOST pointers */
  const specattn_verify_args* verify;     /* HOST [n_target_layers] */
  const void* const* q_host;              /* HOST [n_target_layers] of HOST pointers (bf16) */
  float* const* out_host;                 /* HOST [n_target_layers] of HOST pointers */
  float* const* lse_host;                 /* HOST [n_target_layers] of HOST pointers */
} specattn_step_host_args;

int specattn_verify_step_host(const specattn_step_host_args* args, void* cuda_stream);

/* ========================================================================================
 * A K/V cache held in 4 bits.
 *
 * (No counterpart in the paper, whose cache is 16 bits wide; the operations below serve the same
 * step from a cache of 68 instead of 256 bytes a row.)
 *
 * A row is the 128 values x of one position, KV head and side (kv = 0 keys, 1 values).  It is
 * stored as a scale s and a zero point z in the 16-bit type of the model and a 4-bit code per value:
 *     z = min x      s = (max x - z) / 15, the quotient rounded to binary32, then to 16 bits
 *     c_e = min(15, rint((x_e - z) / s))       (difference and quotient rounded to binary32,
 *                                              rint to even; all codes 0 where s < 2^-126)
 * and stands for s c_e + z.  z is exact, being one of the values; s below 2^-126 is stored as 0.  A
 * row that holds NaN or an infinity, or whose max x - min x overflows binary32, is stored as s = z =
 * NaN, c = 0.
 *   codes:  byte e/2 of a row holds code e in its low and code e + 1 in its high four bits (e even).
 *           Row (page, kv, slot, head) starts at codes + page*stride_page + kv*stride_kv +
 *           slot*stride_slot + head*stride_head (bytes; base 16-byte aligned, strides multiples of 16).
 *   params: s and z, side by side, at params + page*pstride_page + ... (16-bit elements; base
 *           4-byte aligned, strides even).
 * Position i of sequence b lives in page block_table[b * block_table_stride + i / page_size] at slot
 * i % page_size; with block_table == NULL that page is b * block_table_stride + i / page_size.  Unlike
 * the 16-bit pool's, n_pages is required: page ids outside [0, n_pages) are never followed.
 * A layout with the slots of one page and head side by side (stride_slot = 64, stride_head =
 * page_size * 64, and alike for params) lets a scan of everything read whole 32-byte sectors of params.
 * ======================================================================================== */
#define SPECATTN_DTYPE_BF16 0
#define SPECATTN_DTYPE_FP16 1

typedef struct specattn_kv4_cache {
  void* codes;
  void* params;
  int64_t n_pages;
  int64_t stride_page, stride_kv, stride_slot, stride_head;
  int64_t pstride_page, pstride_kv, pstride_slot, pstride_head;
  const int32_t* block_table;
  int64_t block_table_stride;
  int32_t page_size;
  int32_t dtype; /* SPECATTN_DTYPE_*: of params, and of the rows that come in or go out */
} specattn_kv4_cache;

/* specattn_kv4_append -- writes new K/V rows: row t < n_new[b] of sequence b goes to position
 * start[b] + t.  Everything from one token per sequence to whole prompts.
 * specattn_kv4_read   -- the reverse: rows start[b] + t, t < n_new[b], as 16-bit values
 * (s c + z in binary32, rounded to even).  Rows t >= n_new[b] of the buffers are neither read nor
 * written by either.
 * k, v (not looked at where n_tokens == 0): element (b, t, head, e) at b*stride_batch + t*stride_token + head*stride_head + e, 16-byte
 * aligned, strides multiples of 8.  n_new == NULL: n_tokens of every sequence (values beyond
 * [0, n_tokens] are clamped).  status (int32 [batch], optional) is cleared by the call and receives
 * SPECATTN_ROW_BAD_INDEX where a position is negative or beyond the block table or its page id out of range
 * (that row is skipped) and, on append, SPECATTN_ROW_INVALID_VALUE.  No two rows of a call may be written to one
 * place (a page in two sequences' tables, overlapping k or v of a read).
 * Requirements: head_dim == 128; batch and n_kv_heads at most 65535. */
typedef struct specattn_kv4_rows_args {
  uint32_t struct_size;
  int32_t batch;
  int32_t n_tokens;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t reserved; /* 0 */
  specattn_kv4_cache cache;
  void* k;
  void* v;
  int64_t k_stride_batch, k_stride_token, k_stride_head;
  int64_t v_stride_batch, v_stride_token, v_stride_head;
  const int32_t* start; /* [batch] */
  const int32_t* n_new; /* [batch] or NULL */
  int32_t* status;      /* [batch] or NULL */
} specattn_kv4_rows_args;

int specattn_kv4_append(const specattn_kv4_rows_args* args, void* cuda_stream);
int specattn_kv4_read(const specattn_kv4_rows_args* args, void* cuda_stream);

/* specattn_kv4_verify -- specattn_sparse_verify over a cache held in 4 bits.
 *
 * The same operation on the values that the codes stand for: for query row q of KV head hk and the
 * positions i of its list (then the in-flight tail),
 *   s_i = sm_scale * (s_K[i] * sum_e q_e c_K[i,e] + z_K[i] * sum_e q_e)
 *   out_e = sum_i p_i (s_V[i] c_V[i,e] + z_V[i]) / sum_i p_i,  p_i = exp(s_i - max s),
 *   lse   = max s + ln sum_i p_i.
 * An empty list gives out = 0, lse = -inf.  Lists, dense, kv_len, tail_len, sm_scale and n_groups as
 * in specattn_sparse_verify; one query and no list (n_q = 1, dense = 1) is plain decoding.  Scores,
 * sums and outputs are binary32; a weight p_i s_V[i] enters the second product as two 11-bit numbers, 21 bits in all.
 * q is of the cache's dtype, [batch, n_q, n_q_heads, 128], 16-byte aligned; out has the same shape, in
 * that dtype or (out_f32 != 0) binary32, 16-byte aligned; lse binary32 [batch, n_q, n_q_heads].
 * status (int32 [batch], optional) is written by the call: SPECATTN_ROW_BAD_INDEX where a listed
 * position is outside [0, kv_len[b]), a position beyond the block table or its page id out of range
 * (such entries are read from position 0 / page 0 instead), else 0.
 * Positions whose row holds NaN make the rows that attend them NaN; rows that no list names, masked tail rows
 * and the rest of the last page are not looked at.  Values are summed before the division by sum p_i: their magnitude
 * times the number of positions has to stay within binary32.  Such a weight is off
 * by at most 2^-21 of itself or 2^-29 of the largest scale of the rows that the query has met, whichever is more (scales below 2^-122
 * count as 2^-122 there).
 * out must not overlap q.
 * Requirements: head_dim == 128; n_q * (n_q_heads / n_kv_heads) <= 64; batch * n_kv_heads <= 2048; lists
 * and, where dense, block_table_stride * page_size of at most 2^23 positions; and (SPECATTN_ERR_UNSUPPORTED otherwise)
 * no negative stride, the codes of one head within 64 GB and its params within 16 GB of their first
 * (n_pages * stride_page + stride_kv + page_size * stride_slot).
 * flags: SPECATTN_VERIFY_ENGINE_MMA_SYNC or SPECATTN_VERIFY_ENGINE_TCGEN05 forces one of two implementations of the same
 * operation; TCGEN05 runs 25 to 48 query rows (SPECATTN_ERR_UNSUPPORTED otherwise).  With neither the library picks by the
 * sizes of the call: MMA_SYNC for lists, and where dense for block tables with little room.  A caller of 33 rows or more whose lists
 * hold well over 1024 positions an SM in all does better to force TCGEN05, one whose contexts are far shorter than the block table
 * MMA_SYNC.  Results agree within the tolerance of the operation either way.
 * workspace: specattn_kv4_verify_workspace_bytes() bytes, 256-byte aligned, no preparation and no
 * state between calls; two calls that may overlap on the GPU need separate ones.
 * (The call signals programmatic launch completion early: it does not count as the launch in front of a
 * specattn_sparse_verify call with SPECATTN_VERIFY_LISTS_STABLE.) */
typedef struct specattn_kv4_verify_args {
  uint32_t struct_size;
  int32_t batch;
  int32_t n_q;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t n_groups;
  int32_t dense;
  specattn_kv4_cache cache;
  const void* q;
  const int32_t* kv_len; /* [batch] */
  const int32_t* idx;    /* [batch, n_groups, idx_stride]; may be NULL where idx_stride == 0 (the tail alone) */
  int64_t idx_stride;
  const int32_t* counts; /* [batch, n_groups] */
  float sm_scale;        /* > 0, or 0 => 1/sqrt(head_dim); negative or NaN is rejected */
  int32_t out_f32;
  void* out;
  float* lse;
  int32_t* status; /* [batch] or NULL */
  void* workspace;
  size_t workspace_bytes;
  int32_t tail_len; /* 0 <= tail_len <= 64 */
  uint32_t flags;   /* SPECATTN_VERIFY_ENGINE_* (TEST_LOSE_ARRIVAL: TEST ONLY, as there), 0 for none */
} specattn_kv4_verify_args;

/* Bytes of workspace for these shapes on the current device (0 on argument error). */
size_t specattn_kv4_verify_workspace_bytes(const specattn_kv4_verify_args* args);
int specattn_kv4_verify(const specattn_kv4_verify_args* args, void* cuda_stream);

/* ========================================================================================
 * Eviction by accumulated attention weight.
 *
 * (Not in the paper, which keeps every row and skips most of them per step.  The draft model's
 * attention maps, which selection reads anyway, say which rows have not been attended for long.)
 *
 * specattn_accumulate: for every draft layer u with draft_probs[u] != NULL, sequence b, group g
 *   scores_out[u,b,g,i] = decay * scores_in[u,b,g,i] + sum over heads h feeding g and s < gamma of
 *                         draft_probs[u][b,h,s,i],       i < min(kv_len[b], L_stride, score_stride)
 * with the sum in binary64, rounded once.  scores_in == NULL counts as zeros and may equal
 * scores_out.  Other entries are left as they were.  Where a contributing probability is negative,
 * NaN or infinite the position gets its old value, undecayed, and row_status[u,b,g] (optional, cleared by
 * the call, for every u) SPECATTN_ROW_INVALID_PROB.
 * Column i of a map is credited to slot i of the list.  Slots are tokens until specattn_evict's moves have been carried out; from then
 * on slot i holds token positions[u,b,g,i], and a map (or a list of specattn_select_topp made from it) has to be in the order of
 * the slots, too.  It is where the draft's own cache has been moved by the same lists (one list, or one for each of its KV heads,
 * as in specattn_move_rows).  A draft that keeps its whole cache gives maps of tokens: the caller gathers them by positions
 * before the call, each head's by the positions of the group that it feeds; nothing here can tell the one from the other.
 * Arrays, limits and alignment of draft_probs, kv_len and head_group as in specattn_select_topp (gamma at most
 * SPECATTN_MAX_ROWS_PER_LIST, batch and, where heads are grouped, batch * n_groups at most 65535);
 * scores are binary32 [n_layers, batch, n_groups, score_stride]. */
typedef struct specattn_accumulate_args {
  uint32_t struct_size;
  int32_t n_layers;
  int32_t batch;
  int32_t n_draft_heads;
  int32_t gamma;
  int32_t n_groups;
  int64_t L_stride;
  const float* const* draft_probs; /* HOST array [n_layers] of device pointers or NULL */
  const int32_t* kv_len;           /* [batch] */
  const int32_t* head_group;       /* HOST [n_draft_heads] or NULL */
  double decay;                    /* finite, >= 0 */
  const float* scores_in;
  float* scores_out;
  int64_t score_stride;
  int32_t* row_status; /* [n_layers, batch, n_groups] or NULL */
} specattn_accumulate_args;

int specattn_accumulate(const specattn_accumulate_args* args, void* cuda_stream);

/* specattn_evict: which rows stay when every sequence gives up all but `budget` of its positions, and
 * which moves close the gaps.  For each list (u, b, g), n = kv_len[b] (clamped to [0, L]):
 *   slot i < n holds token pos(i) = positions[u,b,g,i], or i where positions == NULL; the sequence has
 *   seen seq_len[b] tokens (n where seq_len == NULL).  A slot is protected when pos(i) < n_sink or
 *   pos(i) >= seq_len[b] - n_recent.  The m = min(n, budget) slots that stay are the protected ones, then
 *   those of the highest score; among equals the lower slot stays.  (-0 counts as 0, NaN as -inf.)
 *   Moves: the slots >= m that stay, ascending, go to the slots < m that do not, ascending:
 *   src[u,b,g,j] -> dst[u,b,g,j], j < n_moves[u,b,g] <= min(budget, L - budget).  Entries behind are
 *   left as they were.  No slot is both read and written, so moves may run in any order; rows in front
 *   that stay are not touched, and slots stop being in token order: positions tells it.  (What the draft's maps and the lists made
 *   from them then have to look like: see specattn_accumulate.)
 *   new_len[b] = m, which is the sequence's kv_len once the rows have been moved.
 *   scores_out (optional): the scores after the moves, 0 in slots [m, n) so that tokens appended there
 *   start from nothing; may equal scores.  positions_out (optional, needs positions): likewise, slots
 *   >= m left as they were; may equal positions.
 * All of scores, positions, scores_out and positions_out are [n_layers, batch, n_groups, L].
 * Requirements: 1 <= L <= SPECATTN_MAX_KV_LEN; budget >= 1; n_sink, n_recent >= 0, their sum <= budget;
 * move_stride >= min(budget, L - budget); n_layers * batch * n_groups <= 2^24; new_len must not be kv_len or seq_len. */
typedef struct specattn_evict_args {
  uint32_t struct_size;
  int32_t n_layers;
  int32_t batch;
  int32_t n_groups;
  int64_t L;
  const float* scores;
  const int32_t* kv_len; /* [batch] */
  int32_t budget;
  int32_t n_sink;
  int32_t n_recent;
  int32_t reserved;         /* 0 */
  const int32_t* positions; /* or NULL */
  const int32_t* seq_len;   /* [batch] or NULL */
  int32_t* src;             /* [n_layers, batch, n_groups, move_stride] */
  int32_t* dst;
  int64_t move_stride;
  int32_t* n_moves; /* [n_layers, batch, n_groups] */
  int32_t* new_len; /* [batch] */
  float* scores_out;
  int32_t* positions_out;
} specattn_evict_args;

int specattn_evict(const specattn_evict_args* args, void* cuda_stream);

/* specattn_move_rows: carries out the moves of ONE draft layer's lists in the pools of the target
 * layers that follow it, one launch for up to 32 of them: for every pool, sequence b, move j < n_moves[b,g]
 * and KV head of group g (n_groups == 1: all heads; n_groups == n_kv_heads: head g), K and V:
 *   row(dst[b,g,j]) = row(src[b,g,j]).
 * A pool is any array of rows of row_bytes (a multiple of 16) addressed (page, kv, slot, head) by strides
 * in BYTES (not negative, multiples of 16; base 16-byte aligned): the bf16 pools of specattn_sparse_verify (256) or
 * the codes of a 4-bit cache (64); params, where set, are rows of param_bytes (a multiple of 4) beside
 * them, 4-byte aligned.  No position may be both a source and a destination of a list, nor twice a destination; and no
 * page that a move reads or writes may be in two sequences' tables (a shared prefix has to be copied first).
 * status (int32 [batch], optional) is cleared by the call and receives SPECATTN_ROW_BAD_INDEX where a
 * position is negative or beyond the block table, or its page id outside [0, n_pages) (the move is skipped).
 * Requirements: row_bytes 16 to 4096, param_bytes up to 256, n_kv_heads up to 1024, batch * n_groups up to 65535. */
typedef struct specattn_move_args {
  uint32_t struct_size;
  int32_t n_pools;
  int32_t batch;
  int32_t n_groups;
  int32_t n_kv_heads;
  int32_t page_size;
  int64_t n_pages;
  void* const* pools; /* HOST [n_pools] */
  int64_t row_bytes;
  int64_t stride_page, stride_kv, stride_slot, stride_head;
  void* const* params; /* HOST [n_pools] or NULL */
  int64_t param_bytes;
  int64_t pstride_page, pstride_kv, pstride_slot, pstride_head;
  const int32_t* block_table; /* [batch, block_table_stride], or NULL: contiguous, as in verify */
  int64_t block_table_stride;
  const int32_t* src; /* [batch, n_groups, move_stride] */
  const int32_t* dst;
  int64_t move_stride;
  const int32_t* n_moves; /* [batch, n_groups] */
  int32_t* status;        /* [batch] or NULL */
} specattn_move_args;

int specattn_move_rows(const specattn_move_args* args, void* cuda_stream);

/* Text for a SPECATTN_ERR_* return code (static storage, never NULL). */
const char* specattn_status_string(int code);

/* Number of kernels this library has launched in the calling process since load (for
 * accounting in benchmarks); thread-safe. */
int64_t specattn_kernel_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* SPECATTN_H_ */
