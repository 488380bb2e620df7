/*
 * criticalkv.h -- C ABI of the CriticalKV prefill-time KV-cache compression step for NVIDIA B200 (sm_100a).
 *
 * The library implements one layer-level operation of "Optimizing KV Cache Eviction from an Output Perturbation
 * Perspective": score every cached KV entry of every head, keep a budgeted subset with the paper's two-stage
 * perturbation-constrained rule, and compact K/V.  The three entry points follow the paper's problem statement
 * (Algorithm 1 inputs: budget b, query state, K, V, W^O, alpha; Algorithm 2 inputs: Q, K, V, window size):
 *
 *   criticalkv_score    steps 1-2   window attention (Algorithm 2) and the projected value-row norm (Algorithm 1)
 *   criticalkv_select   steps 3-4   scores per KV head, budgets, two-stage top-k (Algorithm 1)
 *   criticalkv_compact  step  5     gather of the retained rows (Algorithm 1, the step that appends the selected entries to the retained cache)
 *
 * Conventions
 *   - Every data pointer is a DEVICE pointer unless the argument is documented as host memory.  The caller owns all
 *     buffers, including the workspace; the library allocates device memory only in criticalkv_create (one status
 *     word).
 *   - Calls only enqueue work on the given CUDA stream (a cudaStream_t passed as void*, NULL = legacy default stream)
 *     and return; they never synchronise, except criticalkv_device_status and criticalkv_compress_host.
 *   - Return value: a criticalkv_status.  Argument errors are found on the host before any launch.  A device-side
 *     anomaly (a bounded wait that ran out) sets the handle's device status word; kernels still terminate.
 *   - Identical inputs give bit-identical outputs (no order-dependent floating-point atomics).
 *   - Data pointers must be 16-byte aligned; strides (in elements) must keep every row 16-byte aligned.
 *   - One handle per host thread / stream.
 *
 * Layouts (innermost index contiguous; nb = batch x layers handled by one call)
 *   Qw  [nb, Hq,  w, dh]   the last w query rows of each query head (the observation window)
 *   K,V [nb, Hkv, n, dh]   the KV cache; query head h reads KV head h / (Hq/Hkv)
 *   WO  [nbw, Hq, dh, dm]  head h's rows h*dh .. (h+1)*dh-1 of the (Hq*dh) x dm output projection (Eq. 2: o = A V W^O);
 *                          nbw = nb, or 1 when CKV_FLAG_WO_SHARED is set
 *   attn, vnorm [nb, Hq, n] float32
 *   idx [nb, Btot] int32, offsets [nb, Hkv+1] int32, stage [nb, Btot] uint8 (1 = stage 1, 2 = stage 2)
 *   K_out, V_out [nb, Btot, dh], same element type as K, V
 *   Btot = Hkv * budget (uniform), budget (flattened adaptive), or the capacity given by the caller (given budgets).
 */
#ifndef CRITICALKV_H_
#define CRITICALKV_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define CKV_API __attribute__((visibility("default")))
#else
#define CKV_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef struct criticalkv_handle_s* criticalkv_handle;

typedef enum {
  CKV_OK = 0,
  CKV_EINVAL = -1,      /* bad argument (null pointer, shape, budget out of range)            */
  CKV_ENOTSUP = -2,     /* valid request this build does not implement                        */
  CKV_EALIGN = -3,      /* pointer or stride not 16-byte aligned                              */
  CKV_EWORKSPACE = -4,  /* workspace smaller than criticalkv_workspace_bytes reports          */
  CKV_ECUDA = -5,       /* a CUDA runtime/driver call failed (see criticalkv_last_cuda_error) */
  CKV_ETIMEOUT = -6,    /* a bounded device-side wait ran out (read via criticalkv_device_status) */
  CKV_EBOUNDS = -7      /* CKV_FLAG_DEBUG_CHECKS: a kernel met an index, offset or count outside its buffer; the
                           access was skipped (read via criticalkv_device_status)                */
} criticalkv_status;

typedef enum { CKV_F32 = 0, CKV_BF16 = 1 } criticalkv_dtype;
typedef enum { CKV_BUDGET_UNIFORM = 0, CKV_BUDGET_FLAT_ADAPTIVE = 1, CKV_BUDGET_GIVEN = 2 } criticalkv_budget_mode;
/* CKV_NORM_L1: the paper's method.  CKV_NORM_L2: vnorm = ||V W^O_h||_2 (appendix on the distance metric), computed
   through the Gram matrix W^O_h W^O_h^T, d_model / head_dim times fewer flops than the L1 projection. */
typedef enum { CKV_NORM_L1 = 0, CKV_NORM_L2 = 1 } criticalkv_norm;

enum {
  CKV_FLAG_WO_SHARED = 1u << 0,   /* WO has no nb dimension (one projection for the whole call)             */
  CKV_FLAG_FORCE_SIMT = 1u << 1,  /* use the CUDA-core kernels instead of the tensor-core ones (bf16, and
                                     criticalkv_decode of float32 queries on 4-bit pages)                   */
  CKV_FLAG_PROTECT_WINDOW = 1u << 3, /* always keep the last w entries (the observation window): their scores are
                                     raised to the largest float32 in both stages, so they fill stage 1 first and
                                     count against the budget                                                   */
  CKV_FLAG_WO_GROUP_SUM = 1u << 2, /* grouped-query shortcut of step 2: the W^O slices of a KV group are added
                                     (float32, heads ascending, rounded once to the storage type) and each value
                                     row is projected once per KV head.  vnorm then is [nb, Hkv, n] and
                                     c_g = (a_g + eps) * vnorm_g in criticalkv_select.  Hq/Hkv times fewer flops;
                                     not the per-head norm of Algorithm 1 but the norm of the group's summed
                                     projection (the heads of a group share V, so their outputs add in Eq. 2).  */
  CKV_FLAG_SELECT_MULTIPASS = 1u << 5, /* criticalkv_select: always run steps 3-4 as separate kernels (group scores,
                                     budget allocation, two-stage top-k over score arrays in the workspace) even
                                     when a head's scores fit in shared memory and the single-kernel path applies.
                                     Same results bit for bit                                                   */
  CKV_FLAG_SELECT_SINGLE_KERNEL = 1u << 4, /* criticalkv_select: take the single kernel (one CTA per KV head) also for
                                     calls with few heads (nb * Hkv at most half the number of SMs), which by
                                     default run the separate kernels with a thread-block cluster per head: a
                                     layer at a time that is about twice as fast.  Same results bit for bit      */
  CKV_FLAG_SELECT_NO_CLUSTER = 1u << 8, /* criticalkv_select: no thread-block clusters in steps 3-4 (the separate
                                     kernels then give every head one CTA), for contexts where cluster launches are
                                     not wanted.  Same results bit for bit.  criticalkv_select_pages: likewise.
                                     criticalkv_decode: none either, some small calls take two launches then; the sums are
                                     added in another order                                                    */
  CKV_FLAG_DEBUG_CHECKS = 1u << 6, /* device-side checks in criticalkv_select, criticalkv_compact and
                                     criticalkv_gather_positions: every index read from idx / offsets / budgets and
                                     every output position is tested against the bounds the descriptor implies
                                     before it is used; a violation skips that access, sets the status word to
                                     CKV_EBOUNDS and lets the kernel finish (no trap).  Without the flag the same
                                     accesses are skipped silently.  Meant for bring-up of a caller: the stand-in
                                     for a memory checker where none can be run                                  */
  CKV_FLAG_REQUIRE_TENSOR_CORES = 1u << 7 /* criticalkv_score: return CKV_ENOTSUP instead of running the CUDA-core
                                     kernels when a bf16 problem is outside what the tensor-core kernels take
                                     (window attention: w in {16, 32, 64, 128, 256} and a layout a tensor map can
                                     express; they are 20 times faster, so a silent change of path is a
                                     performance cliff; criticalkv_last_path tells which kernels ran)          */
};

/* Problem descriptor (plain data, copied by every call). */
typedef struct {
  int32_t nb;            /* >= 1                                                                        */
  int32_t Hq, Hkv;       /* Hq % Hkv == 0, Hkv <= 64                                                    */
  int32_t dh;            /* head dim: 64 or 128                                                         */
  int32_t dm;            /* model dim, multiple of 8                                                    */
  int32_t n;             /* cached entries per head, >= w                                               */
  int32_t w;             /* observation window (Algorithm 2: n'), 1..256 (criticalkv_diagnose: 1..64)   */
  int32_t pool_k;        /* max-pool kernel, odd, 1..63 (Algorithm 2: maxpooling; 7 in the paper)       */
  int32_t dtype;         /* criticalkv_dtype of Qw, K, V, WO, K_out, V_out                              */
  float scale;           /* logit scale of Eq. 2; <= 0 selects 1/sqrt(dh)                               */
  float alpha;           /* stage split of Algorithm 1 in [0,1]: b' = floor(alpha*b), b'' = b - b'      */
  float eps;             /* Algorithm 1: (A + eps) * norm; the paper uses 1e-4                          */
  int32_t budget_mode;   /* criticalkv_budget_mode                                                      */
  int32_t norm;          /* criticalkv_norm                                                             */
  int64_t budget;        /* UNIFORM: B per KV head (<= n); FLAT_ADAPTIVE: B_total per nb slice
                            (<= Hkv*n); GIVEN: capacity Btot of idx per nb slice (>= sum of budgets)    */
  uint32_t flags;        /* CKV_FLAG_*                                                                  */
  uint32_t reserved;     /* must be 0                                                                   */
  /* Element strides of Qw / K / V for the nb, head and row (token) index; 0 selects the dense default. */
  int64_t q_stride[3];
  int64_t k_stride[3];
  int64_t v_stride[3];
  float adaptive_floor;  /* FLAT_ADAPTIVE only, in [0,1]: every KV head is first guaranteed
                            floor(adaptive_floor * budget / Hkv) entries, the rest of the budget goes to the
                            flattened top-k, and a head's budget is capped at n.  0 in the paper's settings.   */
  uint32_t reserved2;    /* must be 0                                                                   */
  const int32_t* valid_from; /* NULL, or device int32 [nb,Hkv]: KV head g of slice b holds its entries right-aligned,
                            rows i < valid_from[b,g] of K and V are padding (0 <= valid_from <= n - w).  Padding
                            is invisible to the window queries, gets attn = 0 and the scores a = c = -1, below
                            every real entry, so it is selected only if a head's budget exceeds its n -
                            valid_from real entries (the caller's to avoid; adaptive allocation never does while
                            budget <= number of real entries).  This is the ragged cache that adaptive budgets
                            leave between the chunks of a chunked prefill.  Not accepted by
                            criticalkv_compress_host and criticalkv_diagnose.                              */
} criticalkv_desc;

/* Create / destroy a handle bound to CUDA device `device`.  create allocates one device status word. */
CKV_API int criticalkv_create(criticalkv_handle* out, int device);
CKV_API int criticalkv_destroy(criticalkv_handle h);

/* Workspace sizes in bytes for score and select (host computation, no CUDA call); compact needs none. */
CKV_API int criticalkv_workspace_bytes(const criticalkv_desc* d, size_t* score_bytes, size_t* select_bytes);

/*
 * Steps 1-2.  attn[nb,Hq,n]: per query head the causal softmax of the w window queries over all n keys (window row
 * j sits at position n-w+j and sees keys i <= n-w+j), averaged over the window and max-pooled along the sequence
 * (Algorithm 2; Eq. 2).  vnorm[nb,Hq,n]: L1 norm of each value row projected through that head's slice of W^O
 * (Algorithm 1, "L1 norm of each row of V W^O"; Theorem 3.3).  The n x dm product is never written to memory.
 * Either output may be NULL to skip that half.  ws: workspace of at least score_bytes, 256-byte aligned.
 */
CKV_API int criticalkv_score(criticalkv_handle h, const criticalkv_desc* d, const void* Qw, const void* K,
                             const void* V, const void* WO, float* attn, float* vnorm, void* ws, size_t ws_bytes,
                             void* stream);

/*
 * Steps 3-4.  Per KV head g: a_g = mean over the group's query heads of attn, c_g = mean of (attn + eps) * vnorm
 * (Algorithm 1), each +, *, / a separately rounded float32 operation, heads summed in increasing order.  Budgets:
 * uniform, flattened top-B_total of a over (g, i) counted per head (Algorithm 2, budget allocation), or read from
 * budgets_in[nb,Hkv] (device).  Then stage 1 keeps the b' largest a_g, stage 2 the b'' largest c_g among the rest
 * (Algorithm 1); ties go to the lower index; idx is ascending inside each head's segment
 * [offsets[g], offsets[g+1]).  stage may be NULL.  With given budgets whose sum is below the capacity the tail of
 * idx is left untouched; budgets outside [0, n] or beyond the capacity are clipped and flagged in the status word.
 * Three implementations give the same bits: one kernel with a CTA per head (default when nb * Hkv exceeds half the
 * number of SMs), separate kernels with a thread-block cluster per head (default for fewer heads, i.e. a layer at a
 * time), separate kernels with a CTA per head (heads too long for the other two); CKV_FLAG_SELECT_* override the
 * choice and criticalkv_last_path reports it.
 */
CKV_API int criticalkv_select(criticalkv_handle h, const criticalkv_desc* d, const float* attn, const float* vnorm,
                              const int32_t* budgets_in, int32_t* idx, int32_t* offsets, uint8_t* stage, void* ws,
                              size_t ws_bytes, void* stream);

/*
 * The two front steps of criticalkv_select on their own, for a layer whose KV heads are spread over several GPUs
 * (each GPU holds some KV heads, their query heads and their rows of W^O).  Uniform budgets need nothing from other
 * GPUs.  The flattened adaptive allocation (Algorithm 2, budget allocation) ranks the group attention scores of ALL
 * heads of the layer, so each GPU
 *   1. criticalkv_score on its heads, then criticalkv_group_scores: a_out[nb,Hkv_local,n] (and c_out, which may be
 *      NULL) from attn and vnorm exactly as criticalkv_select computes them;
 *   2. all-gathers a over the head axis (the caller's collective: Hkv*n floats per layer);
 *   3. criticalkv_allocate_budgets with the descriptor of the WHOLE layer (Hkv, budget = B_total, CKV_BUDGET_FLAT_
 *      ADAPTIVE; Hq, dh, dm only need to be consistent): budgets_out[nb,Hkv] int32, identical on every GPU;
 *   4. criticalkv_select with its local descriptor in CKV_BUDGET_GIVEN mode and its slice of the budgets.
 * The result equals, head for head, that of one GPU holding the whole layer.  All pointers are device memory,
 * a/attn/vnorm 16-byte aligned; neither call needs a workspace.
 */
CKV_API int criticalkv_group_scores(criticalkv_handle h, const criticalkv_desc* d, const float* attn,
                                    const float* vnorm, float* a_out, float* c_out, void* stream);
CKV_API int criticalkv_allocate_budgets(criticalkv_handle h, const criticalkv_desc* d, const float* a,
                                        int32_t* budgets_out, void* stream);

/*
 * Allocation-free variant of criticalkv_select (the paper has no counterpart: this is a packaging of steps 3-4 for
 * callers that cannot provide a workspace).  Some hosts of this library may not allocate device memory at the point
 * where they compress a cache: a serving engine that reserved all of HBM for its own pools at start-up has nothing
 * left for cudaMalloc, and a latency-critical loop cannot afford the device-wide synchronisation an allocation or a
 * free implies.  This entry point therefore takes no workspace: the group scores and per-head budgets go to a fixed
 * array of CKV_STATIC_SCRATCH_BYTES that lives inside the library image (every GPU that loads the library keeps
 * that much memory until the process exits).  Arguments and results are those of criticalkv_select.
 *   - The request must fit: if the select_bytes that criticalkv_workspace_bytes reports exceeds
 *     CKV_STATIC_SCRATCH_BYTES (about nb*Hkv*n > 2^20 scored entries) the call returns CKV_EWORKSPACE, launches
 *     nothing, and criticalkv_last_cuda_error describes the sizes.
 *   - The first call on each device looks up the array's device address (once, with that device current); make that
 *     first call outside any stream capture.  No call allocates or frees device memory.
 *   - All calls, from every handle and stream of the process, share the one array per device.  Nothing is read from
 *     it before this call has written it, so stale contents are harmless, but two calls whose kernels may overlap on
 *     the GPU (different streams) race on it: order them on one stream or with events.
 */
#define CKV_STATIC_SCRATCH_BYTES ((size_t)((8u << 20) + (64u << 10)))
CKV_API int criticalkv_select_static(criticalkv_handle h, const criticalkv_desc* d, const float* attn,
                                     const float* vnorm, const int32_t* budgets_in, int32_t* idx, int32_t* offsets,
                                     uint8_t* stage, void* stream);

/* Step 5.  K_out[nb, r, :] = K[nb, g, idx[nb, r], :] for r in head g's segment, same for V (bit copy). */
CKV_API int criticalkv_compact(criticalkv_handle h, const criticalkv_desc* d, const void* K, const void* V,
                               const int32_t* idx, const int32_t* offsets, void* K_out, void* V_out, void* stream);

/*
 * Companion of criticalkv_compact for chunked prefill (the paper's long-context deployment: the cache is compressed
 * after every prefill chunk and later chunks see [retained entries ; new chunk]).  pos_in[nb,Hkv,n] int32 holds the
 * original token position of every cached entry; pos_out[nb, r] = pos_in[nb, g, idx[nb, r]] keeps them attached to
 * the retained rows.
 */
CKV_API int criticalkv_gather_positions(criticalkv_handle h, const criticalkv_desc* d, const int32_t* pos_in,
                                        const int32_t* idx, const int32_t* offsets, int32_t* pos_out, void* stream);

/* The three calls above back to back on one stream.  ws must hold max(score_bytes, select_bytes). */
CKV_API int criticalkv_compress(criticalkv_handle h, const criticalkv_desc* d, const void* Qw, const void* K,
                                const void* V, const void* WO, const int32_t* budgets_in, float* attn, float* vnorm,
                                int32_t* idx, int32_t* offsets, uint8_t* stage, void* K_out, void* V_out, void* ws,
                                size_t ws_bytes, void* stream);

/*
 * The whole path for callers whose tensors live in HOST memory (pinned memory recommended): Qw, K, V, WO,
 * budgets_in (given budgets only) are host arrays in the dense layouts above, idx [nb,Btot], offsets [nb,Hkv+1],
 * K_out, V_out [nb,Btot,dh] are host arrays that receive the result.  The nb slices are streamed one at a time
 * through two device staging buffers on two internal streams, so that the upload of slice b+1, the kernels of slice b
 * and the download of slice b-1 overlap.  `staging` is DEVICE memory of at least criticalkv_host_staging_bytes(d),
 * 256-byte aligned, owned by the caller; the call allocates no device memory (its first use on a handle creates two
 * streams and three events).  Work starts after everything already queued on `stream`; unlike the other calls this
 * one returns only when the results are in host memory.  Element strides in the descriptor must be 0 (dense).
 */
CKV_API int criticalkv_host_staging_bytes(const criticalkv_desc* d, size_t* bytes);
CKV_API int criticalkv_compress_host(criticalkv_handle h, const criticalkv_desc* d, const void* Qw, const void* K,
                                     const void* V, const void* WO, const int32_t* budgets_in, int32_t* idx,
                                     int32_t* offsets, void* K_out, void* V_out, void* staging,
                                     size_t staging_bytes, void* stream);

/*
 * Perturbation diagnostics of Section 3 for a finished selection (not on the hot path).  For every query head and
 * window row j, with A the causal softmax row of that query and nu = vnorm of the head:
 *   diag[nb,Hq,w,10] = sigma (attention mass of the stage-1 set, Assumption 3.4), retained mass, C = sum_i A_i nu_i,
 *   its parts over stage 1 and stage 2, min_i nu_i, L = ||(A - A') V W^O||_1 (Definition 3.1 with A' of Theorem 3.2),
 *   theta (Theorem 3.3), theta_hat (Theorem 3.5), theta_relax (relaxed bound of the appendix).
 * vnorm is the per-head output of criticalkv_score (CKV_ENOTSUP with CKV_FLAG_WO_GROUP_SUM or w > 64); idx, offsets
 * and stage (required) come from criticalkv_select.  ws: criticalkv_diagnose_workspace_bytes, 256-byte aligned.
 */
#define CKV_DIAG_FIELDS 10
CKV_API int criticalkv_diagnose_workspace_bytes(const criticalkv_desc* d, size_t* bytes);
CKV_API int criticalkv_diagnose(criticalkv_handle h, const criticalkv_desc* d, const void* Qw, const void* K,
                                const void* V, const void* WO, const float* vnorm, const int32_t* idx,
                                const int32_t* offsets, const uint8_t* stage, float* diag, void* ws, size_t ws_bytes,
                                void* stream);

/*
 * ---- Decoding on the compressed cache ---------------------------------------------------------------------------
 *
 * After a prefill has been compressed, decoding reads a cache whose KV heads hold different numbers of rows (adaptive
 * budgets).  The cache is therefore paged per (sequence, KV head): page_table[s, g, :] lists the pages of that head,
 * row i of it is slot i % page_size of page page_table[s, g, i / page_size], and every head has its own length.
 *
 *   criticalkv_rope         rotary positions of new queries and keys (a new token's position is not its row number)
 *   criticalkv_cache_store  writes rows into the pages: new tokens, or the rows a selection kept; quantises them
 *   criticalkv_cache_append the two above in one launch: new tokens' queries and keys rotated, keys and values written
 *   criticalkv_cache_load   reads rows back into a dense tensor, for another compression step
 *   criticalkv_decode       attention of one new token per sequence over the pages
 *   criticalkv_summarise_pages, criticalkv_select_pages
 *                           the pages that score best against the new token's queries, as a page table of their own that
 *                           criticalkv_decode reads: attention over a part of a long cache
 *
 * Page ids outside [0, num_pages), row numbers outside the table and lengths outside [0, max_pages * page_size] never
 * cause an access outside a buffer: such rows are skipped (store, load), treated as absent (decode), lengths are
 * clipped; with CKV_FLAG_DEBUG_CHECKS the status word then reads CKV_EBOUNDS.  The calls may be captured into graphs; the
 * handle, the workspace and all tensors must outlive them.
 */
typedef enum {
  CKV_CACHE_PLAIN = 0, /* pages hold rows in the model's element type (dtype)                                   */
  CKV_CACHE_E4M3 = 1,  /* 8-bit float codes (4 exponent, 3 fraction bits, largest 448), one float32 scale a row   */
  CKV_CACHE_INT8 = 2,  /* 8-bit integer codes in -127..127, one float32 scale a row                               */
  CKV_CACHE_E2M1 = 3   /* 4-bit float codes (2 exponent, 1 fraction bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
                          negatives), two a byte, the earlier element in the low half; an e4m3 scale for every 16
                          elements and a float32 scale a row: dh * 9 / 16 + 4 bytes                               */
} criticalkv_cache_format;
/* A quantised row x[0..dh): s = max(max_i |x_i| / top, 2^-100) with top = 448 or 127, r = 1 / s, code_i = x_i * r
   rounded to nearest even; every operation a separately rounded float32 one (where top * s would overflow, s is the
   float below).  It stands for code_i * s.  A row that holds an infinity or a NaN gets an infinite or NaN scale and
   stands for NaN in every element.
   A 4-bit row: s = max(max_i |x_i| / 2688, 2^-100) (2688 = 448 * 6), r = 1 / s; for each group of 16 elements
   g = e4m3((max of the group * r) * (1/6 as a float)), code_i = e2m1(x_i * (r / g)), 0 where g is 0; roundings to nearest
   even, values beyond 448 and 6 become these, every operation a separately rounded float32 one (where 2688 * s would
   overflow, s is the float below).  It stands for (code_i * g) * s, whose first product is exact.  In a row that holds an
   infinity or a NaN, s is infinite or NaN, g and the codes are 0: it stands for NaN in every element. */

typedef struct {
  int32_t nseq;          /* sequences, >= 0 (0: the calls do nothing)                                           */
  int32_t Hq, Hkv;       /* Hq % Hkv == 0, Hkv <= 64                                                            */
  int32_t dh;            /* head dim: 64 or 128                                                                 */
  int32_t dtype;         /* criticalkv_dtype of the rows given and returned, of q and of out                    */
  int32_t format;        /* criticalkv_cache_format of the pages                                                */
  int32_t page_size;     /* rows a page: 16, 32, 64, 128 or 256                                                 */
  int32_t num_pages;     /* pages in the pool, >= 1                                                             */
  int32_t max_pages;     /* columns of the page table, >= 1; a head holds at most max_pages * page_size rows    */
  uint32_t flags;        /* CKV_FLAG_FORCE_SIMT (criticalkv_decode), CKV_FLAG_SELECT_NO_CLUSTER
                            (criticalkv_decode, criticalkv_select_pages), CKV_FLAG_DEBUG_CHECKS                 */
  float scale;           /* logit scale; <= 0 selects 1/sqrt(dh)                                                */
  uint32_t reserved;     /* must be 0                                                                           */
  int64_t page_stride;   /* elements of k_pages / v_pages from one page to the next, 0 = page_size * dh         */
  void* k_pages;         /* [num_pages, page_size, dh] of dtype (plain), 8-bit codes, or 4-bit codes (dh/2 bytes
                            a row)                                                                              */
  void* v_pages;
  float* k_scale;        /* [num_pages, page_size], quantised formats only                                      */
  float* v_scale;
  const int32_t* page_table; /* [nseq, Hkv, max_pages]; entries behind a head's last page are never read as pages */
  uint8_t* k_group_scale; /* e4m3 [num_pages, page_size, dh/16]; these two are read for CKV_CACHE_E2M1 only      */
  uint8_t* v_group_scale;
} criticalkv_cache;

/* Rotary positions.  The first `rot` elements of every row are rot/2 pairs, (x_i, x_{i+rot/2}) in the half layout and
   (x_{2i}, x_{2i+1}) in the interleaved one; pair i is turned by the angle pos * freq[i] and multiplied by `factor`:
   (a, b) -> factor * (a cos - b sin, b cos + a sin).  Elements rot..dh-1 are copied.  Angles are reduced in float64,
   so far positions lose nothing; a negative position turns back. */
typedef enum { CKV_ROPE_HALF = 0, CKV_ROPE_INTERLEAVED = 1 } criticalkv_rope_layout;
typedef struct {
  int32_t nseq, T;       /* sequences and tokens a sequence, >= 0 (0: nothing to do), product at most 2^31 - 257  */
  int32_t Hq, Hk;        /* heads of q (>= 1) and of k (0: no k)                                                */
  int32_t dh;            /* row length, a multiple of 8, at most 256                                            */
  int32_t rot;           /* rotated elements, even, 2..dh                                                       */
  int32_t dtype;         /* criticalkv_dtype of q, k and the outputs                                            */
  int32_t layout;        /* criticalkv_rope_layout                                                              */
  float factor;          /* finite; 1 except where a long-context scaling also scales the rotated part          */
  uint32_t reserved;     /* must be 0                                                                           */
  /* element strides for the sequence, head and token index; 0 selects the dense default [nseq, H, T, dh] */
  int64_t q_stride[3], k_stride[3], q_out_stride[3], k_out_stride[3];
} criticalkv_rope_desc;

/* q_out = rotated q, k_out = rotated k; pos int32 [nseq, T], freq float64 [rot/2], radians per position.  q_out may be
   q and k_out may be k (same strides); the buffers must not overlap otherwise. */
CKV_API int criticalkv_rope(criticalkv_handle h, const criticalkv_rope_desc* d, const void* q, const void* k,
                            const int32_t* pos, const double* freq, void* q_out, void* k_out, void* stream);

/*
 * Rows into the cache.  Source rows K, V [nseq, Hkv, n, dh] (element strides for sequence, head and row in `stride`,
 * NULL or 0 entries = dense).  Which rows of head (s, g) are written, in order, behind row start[s, g]:
 *   idx == NULL   rows 0..c-1, c = counts[s] (device int32 [nseq]) or n when counts is NULL;
 *   idx != NULL   rows idx[s, offsets[s,g] .. offsets[s,g+1]), the result of criticalkv_select (idx [nseq, idx_rows],
 *                 offsets [nseq, Hkv+1]); counts must be NULL.
 * lens_out[s, g] (may be NULL, may be `start` itself, and must not overlap anything else that the call reads) = start +
 * rows written, at most max_pages * page_size.  K and V share their strides.  Other rows of the pages keep their
 * contents.  No page may be listed twice among the rows that one call writes.
 */
CKV_API int criticalkv_cache_store(criticalkv_handle h, const criticalkv_cache* c, const void* K, const void* V,
                                   int32_t n, const int64_t* stride, const int32_t* idx, const int32_t* offsets,
                                   int64_t idx_rows, const int32_t* counts, const int32_t* start, int32_t* lens_out,
                                   void* stream);

/*
 * New tokens into the cache: criticalkv_rope on q and k, then criticalkv_cache_store of the rotated k (rounded to dtype in
 * between) and of v, in one launch.  r describes q, k and q_out as for criticalkv_rope (nseq, Hq, Hk = Hkv, dh and dtype
 * those of the cache, k_out_stride 0); v [nseq, Hkv, T, dh] has strides of its own (v_stride[3], NULL or 0 entries = dense).
 * Tokens 0..counts[s]-1 of a sequence (device int32 [nseq]; NULL: all T) go behind row start[s, g] of every head; the others
 * are ignored, their rows of q_out keep their contents.  q_out may be q (same strides); start and lens_out as for
 * criticalkv_cache_store.  Where rot is no multiple of 16 the two calls take less time on the device (a prompt down to 0.28 of it, a token 0.53).
 */
CKV_API int criticalkv_cache_append(criticalkv_handle h, const criticalkv_cache* c, const criticalkv_rope_desc* r,
                                    const void* q, const void* k, const void* v, const int64_t* v_stride, const int32_t* pos,
                                    const double* freq, const int32_t* counts, const int32_t* start, void* q_out,
                                    int32_t* lens_out, void* stream);

/*
 * Rows out of the cache.  K_out, V_out [nseq, Hkv, n, dh] (strides as above).  With align_right == 0 row i of head
 * (s, g) goes to row i for i < min(lens[s,g], n); with align_right == 1 the last min(lens, n) rows end at row n-1,
 * the layout that criticalkv_desc.valid_from = n - lens describes.  Other rows of the outputs keep their contents, or are
 * zeroed with CKV_LOAD_CLEAR added to align_right.
 */
#define CKV_LOAD_CLEAR (1 << 8)
CKV_API int criticalkv_cache_load(criticalkv_handle h, const criticalkv_cache* c, const int32_t* lens, int32_t n,
                                  const int64_t* stride, int32_t align_right, void* K_out, void* V_out, void* stream);

/*
 * Attention of one new token per sequence: for query head h of sequence s, with g = h / (Hq/Hkv) and the L = lens[s, g]
 * rows of that KV head, out[s, h, :] = sum_i softmax_i(scale * q . k_i) v_i and lse[s, h] = log sum_i exp(scale * q .
 * k_i) (lse may be NULL; it is what merging with attention over other keys needs).  A head without rows gives zeros and
 * -infinity; one that has rows but none in an existing page, or only logits of -infinity, gives NaN; rows with infinite or
 * NaN values give results that are not finite (a key that makes a logit -infinity has no weight).  q [nseq, Hq, dh] with element strides q_stride[2] for sequence and head (NULL or 0 = dense); out dense.
 * bf16 queries run on tensor cores: stored 8-bit values enter exactly, sums and the softmax are float32, and a weight
 * enters its product with the values rounded to 16 bits (plain pages) or, times the row's scale, to 22 bits and no finer than
 * 2^-40 of the head's largest such product (8-bit pages; 2^-36 on 4-bit pages, whose code times group scale enters exactly).
 * float32 queries, and CKV_FLAG_FORCE_SIMT, run on CUDA cores, in float32 throughout; on 4-bit pages float32 queries run on
 * tensor cores too, an element as the sum of two halves (its error 2^-23 of it, or 2^-39 of the query's largest element where
 * that is more).  CKV_ENOTSUP when nseq * Hkv * ceil(Hq/Hkv / 8) exceeds 2^26 or, times ceil(max_pages *
 * page_size / 64), 2^31 - 1.  ws: criticalkv_decode_workspace_bytes, 256-byte aligned,
 * needs no initialisation; calls that may overlap on the GPU need workspaces of their own.
 */
CKV_API int criticalkv_decode_workspace_bytes(const criticalkv_cache* c, size_t* bytes);
CKV_API int criticalkv_decode(criticalkv_handle h, const criticalkv_cache* c, const void* q, const int64_t* q_stride,
                              const int32_t* lens, void* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * Attention over a part of a long cache.  A page is summarised by the largest and the smallest value of every channel over
 * its keys (as the pages stand for them, float32); a query is at most as large against any of its keys as the sum over the
 * channels of the larger of query * largest and query * smallest.
 *
 * criticalkv_summarise_pages writes the summaries of the pages that hold rows start[s, g] .. lens[s, g]-1 of every head
 * (start NULL: 0), over all rows that a page holds up to lens: codes int8 [num_pages, 2, dh] (largest, smallest), scales
 * float32 [num_pages], by page id; others keep their contents.  With top the largest magnitude in the page: scale = max(top /
 * 127, 2^-100), r = 1 / scale, largest code = ceil(largest * r), smallest = floor(smallest * r), within -127..127, every
 * operation a float32 one.  A page with an infinity or a NaN gets that scale and codes 0.  A page that several heads or
 * sequences share must hold equally many rows for all of them.
 *
 * criticalkv_select_pages scores the pages of a head and chooses `count` of them: the first `first` and the last `last` ones
 * (first + last <= count), then those with the largest score, the lower page where two are equal.  Score: the group's
 * queries as codes, scale_q = max(max |q| / 127, 2^-100), code = q * (1 / scale_q) rounded to nearest even; sum (exact, of
 * whole numbers) over the channels of max(code * largest, code * smallest), as a float32 times scale_q, times the page's
 * scale; the largest over the query heads of the group.  A score that is NaN counts as the largest, a page id outside the
 * pool as the smallest.  table_out int32 [nseq, Hkv, count]: the ids of the chosen pages in the order of their rows, -1
 * behind them; lens_out [nseq, Hkv]: the rows they hold; chosen (may be NULL) [nseq, Hkv, count]: which pages of the head
 * they are.  criticalkv_decode with page_table = table_out, max_pages = count and lens = lens_out attends to them.  The
 * outputs must not overlap each other or what is read.  CKV_ENOTSUP for Hq/Hkv > 128, max_pages > 32768, nseq * Hkv > 2^26.
 */
CKV_API int criticalkv_summarise_pages(criticalkv_handle h, const criticalkv_cache* c, const int32_t* start,
                                       const int32_t* lens, int8_t* codes, float* scales, void* stream);
CKV_API int criticalkv_select_pages(criticalkv_handle h, const criticalkv_cache* c, const void* q, const int64_t* q_stride,
                                    const int32_t* lens, const int8_t* codes, const float* scales, int32_t count,
                                    int32_t first, int32_t last, int32_t* table_out, int32_t* lens_out, int32_t* chosen,
                                    void* stream);

/*
 * Self-test of the bounded device-side wait every tensor-core kernel uses: launches one CTA that waits, for at most
 * limit_ns nanoseconds, on a barrier nothing will ever signal.  The kernel must give up, write 0 to *observed_device
 * (a device int; 1 would mean the wait claimed success), set the status word to CKV_ETIMEOUT and end normally.
 * limit_ns above CKV_SELFTEST_MAX_WAIT_NS (100 ms) is refused with CKV_EINVAL: no wait of this library may hold an SM
 * for long.
 */
#define CKV_SELFTEST_MAX_WAIT_NS 100000000ull
CKV_API int criticalkv_selftest_bounded_wait(criticalkv_handle h, uint64_t limit_ns, int* observed_device,
                                             void* stream);

/* Reads the device status word (synchronises `stream` first), clears it, and returns it in *out. */
CKV_API int criticalkv_device_status(criticalkv_handle h, void* stream, int* out);

CKV_API const char* criticalkv_status_string(int status);
/* Last CUDA error string (or size diagnostic of criticalkv_select_static) seen by this handle ("" if none); valid
   until the next call on the handle. */
CKV_API const char* criticalkv_last_cuda_error(criticalkv_handle h);
/* Which kernels the last criticalkv_score on this handle launched: bit0 tensor-core window attention,
   bit1 tensor-core projection norm, bit2 CUDA-core window attention, bit3 CUDA-core projection norm,
   bit5: the last criticalkv_select (or
   criticalkv_select_static) ran as the single kernel; bit6: its two-stage top-k ran with a cluster per head;
   bit7: the last criticalkv_decode ran on tensor cores, bit8: on CUDA cores. */
CKV_API int criticalkv_last_path(criticalkv_handle h);
/* Number of kernel launches this handle has issued since it was created. */
CKV_API int64_t criticalkv_launch_count(criticalkv_handle h);

#ifdef __cplusplus
}
#endif
#endif /* CRITICALKV_H_ */
