/*
 * nanospec.h -- C ABI of the NanoSpec draft-step hot path for AMD MI355X (gfx950).
 *
 * The library keeps a context-aware active vocabulary on the GPU, projects draft hidden states
 * onto the active rows of the bf16 LM-head matrix, and selects the top-k draft tokens.  It
 * follows the problem statement of the NanoSpec paper (arXiv 2605.26444):
 *
 *   Eq. 1   z = W_head h                       dense head (the comparison point)
 *   Sec 3.1 z' = W_head[I_t, :] h              sparse head on the active rows only
 *   Eq. 2-3 candidate stream S, appended to at prefill and after every verification
 *   Eq. 4   I_t = Unique(Suffix(S, W_max))     active index set, recency eviction
 *   Alg. 1  SelectDraftTokens(z', I)           top-k over z' mapped back to global ids
 *   Sec 3.3 / appendix                         the same state read as a first-in first-out queue of
 *                                              distinct ids (nanospec_set_stream_policy)
 *   Sec 4.2 softmax over the active set only   log-probabilities with the selection
 *                                              (nanospec_topk_logprob_remap)
 * and, beside the paper: heads on weights kept in 8 bits, and log-probabilities of given tokens with the losses that
 * train a draft (or a policy) on the logits of a head.
 *
 * Conventions
 *   - Token ids are 0-based int32 in [0, V).
 *   - Pointers named d_* are DEVICE pointers, h_* are HOST pointers.  The caller owns every
 *     buffer it passes in; the library owns the state object and frees it in nanospec_destroy.
 *   - `hip_stream` is a hipStream_t passed as void* (NULL = the default stream).  Every call
 *     documented as "asynchronous" only enqueues kernels on that stream: it never synchronises
 *     the host, never allocates and never frees, so it may be recorded into a HIP graph.
 *   - All functions return a nanospec_status; nothing aborts or throws.  Argument errors are
 *     found on the host before anything is launched, in which case nothing is enqueued.
 *   - A state object must not be used from two streams at once.
 *   - Calls without a state run on the device that is current; every device buffer has to be that device's.
 *   - bf16 = upper 16 bits of an IEEE fp32.  Products are accumulated in fp32.
 */
#ifndef NANOSPEC_H_
#define NANOSPEC_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define NANOSPEC_API __attribute__((visibility("default")))
#else
#define NANOSPEC_API
#endif

typedef struct nanospec_state nanospec_state; /* opaque; owns all device-resident state */
typedef int32_t nanospec_status;

enum {
  NANOSPEC_OK = 0,
  NANOSPEC_EINVAL = -1,    /* null pointer, non-positive size, unsupported shape, bad offsets   */
  NANOSPEC_ENOMEM = -2,    /* device or host allocation failed (nanospec_create only)           */
  NANOSPEC_ECAPACITY = -3, /* an input exceeds a capacity fixed at nanospec_create              */
  NANOSPEC_EHIP = -4       /* a HIP runtime call failed                                         */
};

/* Bits reported by nanospec_last_device_error. */
enum {
  NANOSPEC_DEV_BAD_ID = 1 /* an appended or candidate id was outside [0, V); it was ignored     */
};

/* Largest batch (independent sequences per state) supported: per-sequence offsets travel as
 * kernel arguments so that no call needs a host-to-device copy. */
#define NANOSPEC_MAX_BATCH 256

/* Human-readable name of a status code (static storage). */
NANOSPEC_API const char* nanospec_status_string(nanospec_status s);

/* Byte sizes of the device buffers a state with these parameters owns.  Pure host arithmetic
 * (usable without a GPU); nanospec_create allocates exactly these.  For the paper's Llama-3.1-8B
 * setting (V=128256, W_max=3072) the bitmap is ceil(V/32)*4 = 16032 B and the stream ring
 * 3072*4 = 12288 B, the "16 KB" and "12 KB" rows of Table 6; `gathered_bytes_at_cap` is the size
 * the paper's repack buffer would have (window * d * 2; 24 MiB there), which this library never
 * allocates because the gather is fused into the projection. */
typedef struct nanospec_layout {
  int64_t ring_bytes;            /* per sequence: last `window` stream ids, int32                */
  int64_t counter_bytes;         /* per sequence: window multiplicity of every id, uint32[V]     */
  int64_t window_bitmap_bytes;   /* per sequence: 1 bit per id, set iff multiplicity > 0         */
  int64_t topk_bitmap_bytes;     /* per sequence: 1 bit per id, set iff id is in the set T       */
  int64_t ids_bytes;             /* per sequence: ascending active ids, int32[capacity]          */
  int64_t scalars_bytes;         /* per sequence: n, ring position, fill                         */
  int64_t workspace_bytes;       /* whole state: split-K partial logits + top-k candidates       */
  int64_t total_bytes;           /* everything, all sequences                                    */
  int64_t gathered_bytes_at_cap; /* window * d * 2: what a packed copy of the rows would take    */
  int32_t capacity;              /* row stride of ids / logits: max |I_t| rounded up to 64       */
} nanospec_layout;

NANOSPEC_API nanospec_status nanospec_state_layout(int32_t V, int32_t d, int32_t batch, int32_t window,
                                      int32_t topk_cap, int32_t m_cap, int32_t k_cap,
                                      nanospec_layout* out);

/* Create the device-resident state for `batch` independent sequences on the current device.
 *   V         vocabulary size (rows of W_head)            d        hidden size, multiple of 8
 *   window    W_max of Eq. 4                               topk_cap largest |T| per sequence
 *   m_cap     largest number of draft hidden rows per sequence and call
 *   k_cap     largest k of nanospec_topk_remap (<= 64)
 * Limits: batch <= NANOSPEC_MAX_BATCH; min(window + topk_cap, V) <= 262144 (16 top-k chunks); the vocabulary
 * kernels keep three V-bit bitmaps in one workgroup's LDS, which bounds V at about 420 000.
 * Errors: EINVAL (null, a size < 1, d % 8 != 0, a limit above exceeded), ENOMEM, EHIP.
 * Synchronous (allocates).  The state starts empty: stream length 0, T empty, I empty.  The state belongs to
 * the device that is current here; every later call on it returns EINVAL if another device is current. */
NANOSPEC_API nanospec_status nanospec_create(nanospec_state** out, int32_t V, int32_t d, int32_t batch,
                                int32_t window, int32_t topk_cap, int32_t m_cap, int32_t k_cap);
NANOSPEC_API nanospec_status nanospec_destroy(nanospec_state* st);

/* Which reading of the paper's vocabulary the state follows; takes effect at the next nanospec_vocab_init.
 *   NANOSPEC_POLICY_WINDOW (default): Eq. 4 -- the window covers the last W_max entries of the raw stream,
 *       repeats included; a token stays while any of its occurrences is inside the window.
 *   NANOSPEC_POLICY_FIFO: the state management of Sec. 3.3 as the appendix on vocabulary evolution describes
 *       it -- a first-in first-out queue of at most W_max distinct ids.  One call (init, update,
 *       append_unique) pushes, in the order of their first occurrence, the ids that are valid, not members
 *       when the call starts and not repeated inside the call; the oldest members leave first; a member
 *       that is appended again keeps its place.  Ids outside [0,V) are skipped and flagged.
 * Everything else (T, the ascending list, head, selection) is the same.  Errors: EINVAL. */
#define NANOSPEC_POLICY_WINDOW 0
#define NANOSPEC_POLICY_FIFO 1
NANOSPEC_API nanospec_status nanospec_set_stream_policy(nanospec_state* st, int32_t policy);

/* Stream initialisation, Eq. 2 and the first I of Alg. 1: for sequence b the stream becomes
 * ctx_ids[h_ctx_off[b] .. h_ctx_off[b+1]) (only its last `window` ids matter) and the candidate
 * set T becomes topk_ids[h_topk_off[b] .. h_topk_off[b+1]) (duplicates allowed, order
 * irrelevant).  The active set I = Unique(Suffix(S, window)) U T is left on the device as an
 * ascending id list with its count.  The paper appends top-K candidates to the stream itself;
 * that mode is T = empty with those ids appended through ctx/new ids.
 *   d_ctx_ids, d_topk_ids : device int32; may be NULL when every range is empty.
 *   h_ctx_off, h_topk_off : host int32[batch+1], non-decreasing, read before the call returns.
 * Errors: EINVAL (null state/offsets, decreasing offsets), ECAPACITY (a T range > topk_cap).
 * Asynchronous.  Ids outside [0,V) hold their stream position but never become members; they
 * raise NANOSPEC_DEV_BAD_ID. */
NANOSPEC_API nanospec_status nanospec_vocab_init(nanospec_state* st, const int32_t* d_ctx_ids, const int32_t* h_ctx_off,
                                    const int32_t* d_topk_ids, const int32_t* h_topk_off, void* hip_stream);

/* Stream update, Eq. 3 followed by Eq. 4: append new_ids[h_new_off[b] .. h_new_off[b+1]) to the
 * stream of sequence b (zero ids is legal), evict what leaves the window, and bring the
 * ascending active list and its count up to date -- one launch for the whole batch (appends of
 * at most 16 ids that leave T alone patch the list in place, anything else rebuilds it; the
 * result is the same list either way).  If d_topk_ids is not
 * NULL (or h_topk_off is not NULL with all-empty ranges) the set T of every sequence is replaced
 * wholesale; pass both NULL to keep T.  Same argument rules and errors as nanospec_vocab_init.
 * Asynchronous. */
NANOSPEC_API nanospec_status nanospec_vocab_update(nanospec_state* st, const int32_t* d_new_ids, const int32_t* h_new_off,
                                      const int32_t* d_topk_ids, const int32_t* h_topk_off, void* hip_stream);

/* Stream update with the candidate set built on the device, Eq. 3 for C_draft (Sec. 3.2: every distinct
 * token id that occurs in the step's draft tree, accepted or not): for sequence b the ids
 * d_cand_ids[b*cand_stride .. +cand_per_seq) -- typically the [M][k] output of nanospec_topk_remap of the
 * same state, passed without a host round trip -- are de-duplicated and appended to the stream in
 * ascending id order (the paper leaves the order of tuple(set) open), then Eq. 4 as in
 * nanospec_vocab_update.  The number of ids appended is known only on the device.  Entries equal to -1
 * (top-k padding) are skipped; other ids outside [0,V) are skipped and raise NANOSPEC_DEV_BAD_ID.  T is kept.
 * The same call finishes Eq. 2 on the device: after nanospec_vocab_init with the prompt, pass the [L][K_pre]
 * output of nanospec_dense_topk over the prefill logits (the tail of S^(0) is a de-duplicated union too).
 *   d_cand_ids : device int32 [batch][cand_stride]; cand_per_seq is bounded by the LDS of one workgroup:
 *                39776 - 12 * ceil(V/128) entries (27 752 at V = 128256); at least m_cap * k_cap.
 * Errors: EINVAL (null, negative, stride < count), ECAPACITY (cand_per_seq above that bound).  Asynchronous; takes no host integers that
 * change from step to step, so one recorded HIP graph of a whole draft step can be replayed indefinitely. */
NANOSPEC_API nanospec_status nanospec_vocab_append_unique(nanospec_state* st, const int32_t* d_cand_ids,
                                                          int32_t cand_per_seq, int64_t cand_stride, void* hip_stream);

/* Borrowed device views of the active vocabulary, valid until nanospec_destroy; contents are
 * valid in stream order after the last init/update.
 *   *d_ids : int32[batch][capacity], row b holds I of sequence b ascending in [0, n_b)
 *   *d_n   : int32[batch]            |I| per sequence
 *   *capacity : row stride (also the row stride of the logits of nanospec_sparse_head). */
NANOSPEC_API nanospec_status nanospec_vocab_view(const nanospec_state* st, const int32_t** d_ids, const int32_t** d_n,
                                    int32_t* capacity);

/* Sparse head, Eq. 1 restricted to the active rows (Sec. 3.1):
 *   logits[b][m][j] = sum_c W[ids_b[j]][c] * H[b][m][c]   for j < n_b, fp32 accumulation.
 *   d_W_bf16  : bf16 [V][d] row-major by token id          d_H_bf16 : bf16 [batch][M][d]
 *   d_logits  : fp32 [batch][M][capacity]; entries j >= n_b are unspecified.
 * The rows are gathered inside the projection; no packed copy of them is made.  The result for a
 * given (W row, H row) pair does not depend on j, on n or on the other active ids.
 * Errors: EINVAL (null, M < 1), ECAPACITY (M > m_cap).  Asynchronous. */
NANOSPEC_API nanospec_status nanospec_sparse_head(nanospec_state* st, const void* d_W_bf16, const void* d_H_bf16, int32_t M,
                                     float* d_logits, void* hip_stream);

/* The paper's own system design as a variant of the head (Sec. 3.3 "Avoiding sparse computation via asynchronous
 * gathering"; Alg. 1 Gather_Async; the weight-gather row of Table 4; the repacked-weights row of Table 6): a
 * pre-allocated packed buffer of `capacity` rows holds a copy of every active row of W_head; after a vocabulary
 * update only the rows of ids that entered the active set are copied in, and the head is a dense product on
 * the packed buffer.  Slots are stable (an id keeps its slot while it stays active; an entering id takes the
 * lowest free slot), and the logits still come out in the layout of nanospec_sparse_head (column j = j-th
 * active id ascending), so nanospec_topk_remap / nanospec_topk_logprob_remap apply unchanged, ties by lower id
 * included.  One sequence per state (batch == 1).
 *   nanospec_packed_bytes  : device bytes nanospec_packed_enable allocates (capacity*d*2 for the rows -- 24 MiB at
 *                            the paper's W_max = 3072, d = 4096 -- plus V*4 + 20*capacity bytes of slot tables).
 *   nanospec_packed_enable : allocate and clear them.  Synchronous; idempotent.  Errors: EINVAL (batch != 1), ENOMEM, EHIP.
 *   nanospec_packed_gather : bring the buffer in line with the current active list: free the slots of ids that
 *                            left, give every id without a slot one, copy those rows W[id] -> buffer[slot], refresh
 *                            the slot -> column map.  Two launches on `hip_stream`, which may be a second stream
 *                            running beside the draft backbone; the caller orders it after the vocabulary call
 *                            and before nanospec_packed_head with events (the paper's dual-stream pipeline).  The
 *                            first call after nanospec_vocab_init, a T replacement or a long append copies many
 *                            rows, a decoding step a handful.  Asynchronous.  Errors: EINVAL (not enabled), EHIP.
 *   nanospec_packed_head   : logits as nanospec_sparse_head, computed from the packed buffer (W_head is not
 *                            touched).  Asynchronous.  Errors: EINVAL, ECAPACITY (M > m_cap).
 *   nanospec_packed_view   : borrowed device views for inspection: the row buffer bf16 [capacity][d], the id
 *                            held by each slot (-1 free), each slot's logit column (-1 none), and two counters
 *                            {slots that may hold a row, rows copied by the last gather}. */
NANOSPEC_API int64_t nanospec_packed_bytes(const nanospec_state* st);
NANOSPEC_API nanospec_status nanospec_packed_enable(nanospec_state* st);
NANOSPEC_API nanospec_status nanospec_packed_gather(nanospec_state* st, const void* d_W_bf16, void* hip_stream);
NANOSPEC_API nanospec_status nanospec_packed_head(nanospec_state* st, const void* d_H_bf16, int32_t M, float* d_logits,
                                                  void* hip_stream);
NANOSPEC_API nanospec_status nanospec_packed_view(const nanospec_state* st, const void** d_buf, const int32_t** d_slot_id,
                                                  const int32_t** d_out_pos, const int32_t** d_counts);

/* Several sequences in one state (multi-sequence serving; Sec. 4.6 states only that the method's per-sequence cost
 * adds up over the batch): sequences drawing from one token distribution hold many of the same ids.  The lists split
 * the active sets: an id held by at least `min_share` of the sequences is a shared row, listed once; every other id
 * stays on a per-sequence list, and every (sequence, active id) pair is covered by exactly one part.  The head gives the
 * logits of nanospec_sparse_head, in its layout, so that nanospec_topk_remap / nanospec_topk_logprob_remap apply
 * unchanged.  How it computes them is chosen for speed, with batch * capacity the number of pairs there is room for:
 *   - M <= 4, d >= 2048, batch * capacity >= 196608: from the split -- shared rows fetched once and multiplied with the
 *     hidden rows of all sequences, the others per sequence;
 *   - else M <= 16, batch * capacity >= 40960: as nanospec_union_build found the overlap, from the split where the
 *     sequences hold nearly the same ids, else every list whole;
 *   - else as nanospec_sparse_head, whose launch order has sequences find the rows they share in cache; min_share and
 *     shared_cap then shape the lists only.
 *   nanospec_union_bytes  : device bytes nanospec_union_enable allocates for the given shared_cap (-1: bad argument).
 *   nanospec_union_enable : allocate and clear the lists.  min_share: 0 = max(2, batch/8).  shared_cap: room on the
 *                           shared list, a multiple of 64 in [64, capacity], 0 = capacity; when more ids qualify the
 *                           lowest shared_cap are shared and the others stay per sequence.  Synchronous; once per
 *                           state.  Errors: EINVAL (bad arguments, already enabled), ENOMEM, EHIP.
 *   nanospec_union_build  : rebuild the lists from the current vocabulary state (two launches); it needs no hidden
 *                           states, so it may run beside the draft backbone.  Asynchronous.  Errors: EINVAL (not enabled), EHIP.
 *   nanospec_union_head   : d_logits fp32 [batch][M][capacity] as nanospec_sparse_head (entries j >= n_b
 *                           unspecified), from d_W_bf16 [V][d] and d_H_bf16 [batch][M][d].  Call after a vocabulary call
 *                           and the nanospec_union_build that follows it: where it works from the lists they are those of
 *                           the last build, where it does not it reads the active sets themselves, so that a
 *                           vocabulary call between build and head leaves the two out of step.  Two calls on one state
 *                           must not overlap.  Asynchronous.  Errors: EINVAL, ECAPACITY (M > m_cap), EHIP.
 *   nanospec_union_view   : borrowed device views for inspection: shared ids [shared_cap] and their number
 *                           (first entry of d_shared_n), shared_pos [batch][shared_cap] (column or -1), rest ids
 *                           and columns [batch][capacity], rest_n [batch]; any pointer may be NULL. */
NANOSPEC_API int64_t nanospec_union_bytes(const nanospec_state* st, int32_t shared_cap);
NANOSPEC_API nanospec_status nanospec_union_enable(nanospec_state* st, int32_t min_share, int32_t shared_cap);
NANOSPEC_API nanospec_status nanospec_union_build(nanospec_state* st, void* hip_stream);
NANOSPEC_API nanospec_status nanospec_union_head(nanospec_state* st, const void* d_W_bf16, const void* d_H_bf16, int32_t M,
                                                 float* d_logits, void* hip_stream);
NANOSPEC_API nanospec_status nanospec_union_view(const nanospec_state* st, const int32_t** d_shared_ids, const int32_t** d_shared_n,
                                                 const int32_t** d_shared_pos, const int32_t** d_rest_ids,
                                                 const int32_t** d_rest_pos, const int32_t** d_rest_n, int32_t* shared_cap,
                                                 int32_t* min_share);

/* Draft-token selection, SelectDraftTokens(z', I) of Alg. 1 with the operator T_K of Sec. 3.2:
 * for every (b, m) the k largest of logits[b][m][0..n_b), ordered by value descending then global
 * id ascending (+0 and -0 tie), written as global ids and values.  Slots beyond n_b get id -1
 * and value -inf.  NaN logits are not supported.
 *   d_out_ids : int32 [batch][M][k]       d_out_vals : fp32 [batch][M][k] (may be NULL)
 * Errors: EINVAL, ECAPACITY (M > m_cap or k > k_cap).  Asynchronous. */
NANOSPEC_API nanospec_status nanospec_topk_remap(nanospec_state* st, const float* d_logits, int32_t M, int32_t k,
                                    int32_t* d_out_ids, float* d_out_vals, void* hip_stream);

/* Draft-token selection with the draft distribution renormalised over the active vocabulary (Sec. 4.2
 * attributes the acceptance gain on context-heavy tasks to exactly this renormalisation; tree-style
 * drafters rank their nodes by these log-probabilities): ids and order as nanospec_topk_remap, values
 *   logprob[b][m][r] = z_r - log(sum_{j < n_b} exp(logits[b][m][j])),
 * fp32, the sum taken after subtracting the row maximum, partial sums added in a fixed order (the
 * result is reproducible bit for bit).  Slots beyond n_b get id -1 and -inf.
 *   d_out_logprob : fp32 [batch][M][k], required.
 * Errors: EINVAL, ECAPACITY (M > m_cap or k > k_cap).  Asynchronous. */
NANOSPEC_API nanospec_status nanospec_topk_logprob_remap(nanospec_state* st, const float* d_logits, int32_t M, int32_t k,
                                                         int32_t* d_out_ids, float* d_out_logprob, void* hip_stream);

/* Dense full-vocabulary head, Eq. 1: logits[m][v] = sum_c W[v][c] * H[m][c] for all v < V.
 *   d_logits : fp32 [M_total][V].  Stateless.  Errors: EINVAL (null, sizes < 1, d % 8 != 0).
 * Asynchronous. */
NANOSPEC_API nanospec_status nanospec_dense_head(const void* d_W_bf16, const void* d_H_bf16, int32_t V, int32_t d,
                                    int32_t M_total, float* d_logits, void* hip_stream);

/* Top-k over dense logits (the selection step of the full-vocabulary comparison point):
 * rows [M_total][V], ids are the column indices; same ordering rule as nanospec_topk_remap.
 *   d_workspace : device scratch of at least nanospec_dense_topk_workspace(V, M_total, k) bytes.  Asked for whatever
 *                 M_total is, also where the rows are selected without it.
 * Errors: EINVAL (null, sizes < 1, k > 64), ECAPACITY (workspace too small).  Asynchronous. */
NANOSPEC_API int64_t nanospec_dense_topk_workspace(int32_t V, int32_t M_total, int32_t k);
NANOSPEC_API nanospec_status nanospec_dense_topk(const float* d_logits, int32_t V, int32_t M_total, int32_t k,
                                    int32_t* d_out_ids, float* d_out_vals, void* d_workspace,
                                    int64_t workspace_bytes, void* hip_stream);

/* The same selection for callers that cannot allocate device memory -- code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc: no workspace argument; the per-chunk candidates go to a
 * fixed 4 MiB device array inside the library (one per GPU, held until the process ends, its address looked
 * up on the first call on each device).  The call allocates and frees nothing.  Output as
 * nanospec_dense_topk, bit for bit.  Every call on a GPU shares that GPU's array: calls that overlap on one
 * GPU (two streams, two threads) race and must be serialised by the caller; calls in stream order need no
 * clearing in between.
 * Errors: EINVAL (as nanospec_dense_topk), ECAPACITY (nanospec_dense_topk_workspace(V, M_total, k) above
 * nanospec_dense_topk_static_limit() = 4 MiB, e.g. more than 5957 rows at V = 128256, k = 10), EHIP.
 * Asynchronous. */
NANOSPEC_API int64_t nanospec_dense_topk_static_limit(void);
NANOSPEC_API nanospec_status nanospec_dense_topk_static(const float* d_logits, int32_t V, int32_t M_total, int32_t k,
                                                        int32_t* d_out_ids, float* d_out_vals, void* hip_stream);

/* Heads on 8-bit weights: the bytes of W_head bound the heads above, 8 bits halve them.  Every row is kept as int8 with a
 * scale of its own,
 *   a = max_c |x_c|, scale = a / 127, q_c = 127 x_c / a rounded to the nearest integer, ties to even (|q| <= 127),
 * the quotient rounded once: q is what exact arithmetic on the bf16 values gives.  A row of zeros has q = 0 and scale 0, a row that
 * holds an infinity or a NaN q = 0 and scale NaN (all logits it meets are NaN).
 *   nanospec_quantize_rows : d_Q int8 [rows][d] and d_scale fp32 [rows] from d_X bf16 [rows][d]; of the weights, once.
 *   nanospec_dense_head_i8 : logits[m][v] = scale_H[m] scale_W[v] sum_c qH[m][c] qW[v][c] for all v < V, where qH, scale_H are the
 *                            hidden rows d_H_bf16 [M_total][d] quantized by the call in the same way (a scale per token) and
 *                            qW, scale_W the weights' (a scale per vocabulary row).  The sum is taken in 32-bit integers and is
 *                            exact; it is rounded to fp32 and multiplied with the two scales: logits do not depend on the kernel that
 *                            ran.  Layout as nanospec_dense_head.
 *   nanospec_sparse_head_i8: the same on the active rows, layout as nanospec_sparse_head: d_H_bf16 [batch][M][d] -> d_logits fp32
 *                            [batch][M][capacity]; entries j >= n_b are left as they were.  V and d are the state's.
 *   d_workspace : device scratch of at least nanospec_head_i8_workspace(rows, d) bytes, rows = M_total or batch * M (-1: sizes out
 *                 of range), 256-byte aligned; asked for whatever the sizes.  Calls that may overlap (two streams, two captured
 *                 graphs) must not share one.
 * Limits: d a multiple of 16 and at most 133136 (the sum fits 32 bits); V * d and rows * d below 2^32; at most 2^24 hidden rows;
 * d_W_i8, d_Q, d_H_bf16 and d_X_bf16 16-byte aligned.
 * Errors: EINVAL (null, sizes < 1, a limit exceeded), ECAPACITY (M > m_cap, workspace too small), EHIP.  Asynchronous. */
NANOSPEC_API nanospec_status nanospec_quantize_rows(const void* d_X_bf16, int64_t rows, int32_t d, int8_t* d_Q, float* d_scale,
                                                    void* hip_stream);
NANOSPEC_API int64_t nanospec_head_i8_workspace(int32_t rows, int32_t d);
NANOSPEC_API nanospec_status nanospec_dense_head_i8(const int8_t* d_W_i8, const float* d_W_scale, const void* d_H_bf16, int32_t V,
                                                    int32_t d, int32_t M_total, float* d_logits, void* d_workspace,
                                                    int64_t workspace_bytes, void* hip_stream);
NANOSPEC_API nanospec_status nanospec_sparse_head_i8(nanospec_state* st, const int8_t* d_W_i8, const float* d_W_scale,
                                                     const void* d_H_bf16, int32_t M, float* d_logits, void* d_workspace,
                                                     int64_t workspace_bytes, void* hip_stream);

/* Rows of logits with a token each: what the calls below work on.  The struct is read before they return.
 *   d_logits      : [rows][ld] of `type`, columns 0 .. V-1 (those of nanospec_dense_head with ld = V; of nanospec_sparse_head with
 *                   ld = V = capacity, rows = batch * M).
 *   d_tokens      : int32 [rows], global ids.
 *   d_ids, d_n    : NULL: column j is id j.  Else the active sets, as nanospec_vocab_view gives them: row r's columns are the
 *                   ids d_ids[(r / rows_per_list) * V + j] for j < d_n[r / rows_per_list], ascending (rows_per_list = M, a list and
 *                   a count for every M rows); the distribution is renormalised over them, as in nanospec_topk_logprob_remap.
 *                   Columns behind are neither read nor written.
 * A logit of -inf has probability 0.  A token has no probability if it has no column (padding: whatever the row's columns hold) or if
 * its logit is -inf.  Where the token has a column, a NaN or +inf among the row's columns makes the row's results NaN. */
#define NANOSPEC_F32 0
#define NANOSPEC_BF16 1
typedef struct nanospec_logit_rows {
  const void* d_logits;
  const int32_t* d_tokens;
  const int32_t* d_ids;
  const int32_t* d_n;
  int64_t ld;            /* row stride in elements, >= V */
  int32_t type;          /* NANOSPEC_F32 or NANOSPEC_BF16 */
  int32_t rows;
  int32_t V;             /* columns; row stride of d_ids */
  int32_t rows_per_list; /* hidden rows per active set; ignored without d_ids */
} nanospec_logit_rows;

/* Log-probabilities of given tokens (a verifier's or a reference model's view of an answer; the draft's own probabilities of what
 * it proposed, which rejection sampling needs):
 *   logprob[r] = z_r[token] - log sum_j exp(z_r[j]), -inf where the token has no column or its logit is -inf.
 * Losses on the logits of a head, each with the gradient of those logits.  With w_r = d_weight[r] (fp32 [rows]; NULL: 1), a
 * row counts if w_r is not 0; rows that do not count are not read, whatever they hold.  log p_r as above, in fp32 -- max and sums -- and
 * 64 bits behind the sums; every sum has a fixed order, so that results are reproducible bit for bit.
 *   nanospec_policy_loss: the clipped policy loss with a KL term,
 *     ratio = exp(log p_r - d_old[r]), gap = d_ref[r] - log p_r, A = d_adv[r],
 *     row_loss[r] = -min(ratio A, clamp(ratio, 1 - clip_low, 1 + clip_high) A) + kl_beta (exp(gap) - gap - 1),
 *     loss = sum of w_r row_loss[r] over the rows that count (a mean over tokens or answers is a matter of the weights).
 *     d_ref may be NULL if kl_beta is 0.  A row whose token has no probability, or one that is 0 in 64 bits (a log-probability
 *     below -745, of which ratio and KL term take the exponential), has row_loss 0 and no gradient.  d_old may be -inf: the ratio
 *     is infinite then, and its product with an advantage of 0 is 0.
 *   nanospec_preference_loss: the preference loss on `pairs` pairs of answers.  Answer q covers rows h_off[q] .. h_off[q+1), pair p
 *     is answer 2p, the chosen one, and 2p + 1, the rejected one; rows outside h_off[0] .. h_off[2 pairs) do not count;
 *     S_q = sum of w_r (log p_r - d_ref[r]) (d_ref NULL: 0; every finite log p_r counts, also that of a token masked with a finite
 *     value; a row whose token has no probability adds nothing and has no gradient),
 *     margin[p] = beta (S_2p - S_2p+1), loss = mean over p of -(1 - smoothing) log sigma(margin) - smoothing log sigma(-margin),
 *     a term without its factor being 0.  d_ref may be -inf (no probability under the reference): the margin is infinite then.
 *     h_off: host int32 [2 pairs + 1], non-decreasing, within 0 .. rows, read before the call returns; 2 pairs <= NANOSPEC_MAX_BATCH.
 *   d_loss fp32 [1]; d_row_loss [rows], d_margin [pairs], d_logprob [rows]: fp32, each may be NULL.  row_loss and logprob of rows that
 *     do not count are 0.
 *   d_grad : NULL: none.  Else [rows][ld_grad] of grad_type: grad_scale * dloss/dz for every row and its live columns, zeros in rows
 *     that do not count.  It may be the logits' own memory if type and stride are the same, and must not share their range of addresses else.
 *     No other output may share memory with an input.
 *   d_workspace : device scratch of at least nanospec_loss_workspace(rows, V) bytes (-1: sizes out of range), 256-byte aligned; what is
 *     enough for some rows and columns is enough for fewer.  Calls that may overlap must not share one.
 * Limits: rows <= 2^22, rows * ld below 2^60, V <= 2^30; logits and gradients aligned to their type.  Errors: EINVAL (null, sizes < 1, ld < V, an unknown type, d_ids without d_n or
 * the other way round, clip_low or clip_high negative, kl_beta != 0 without d_ref, smoothing outside [0, 1], a NaN among these, bad
 * offsets), ECAPACITY (workspace too small, 2 pairs > NANOSPEC_MAX_BATCH), EHIP.  Asynchronous. */
NANOSPEC_API int64_t nanospec_loss_workspace(int32_t rows, int32_t V);
NANOSPEC_API nanospec_status nanospec_token_logprob(const nanospec_logit_rows* rows, float* d_logprob, void* d_workspace,
                                                    int64_t workspace_bytes, void* hip_stream);
NANOSPEC_API nanospec_status nanospec_policy_loss(const nanospec_logit_rows* rows, const float* d_old, const float* d_ref,
                                                  const float* d_adv, const float* d_weight, float clip_low, float clip_high,
                                                  float kl_beta, float* d_loss, float* d_row_loss, float* d_logprob, void* d_grad,
                                                  int32_t grad_type, int64_t ld_grad, float grad_scale, void* d_workspace,
                                                  int64_t workspace_bytes, void* hip_stream);
NANOSPEC_API nanospec_status nanospec_preference_loss(const nanospec_logit_rows* rows, const int32_t* h_off, int32_t pairs,
                                                      const float* d_ref, const float* d_weight, float beta, float smoothing,
                                                      float* d_loss, float* d_margin, float* d_logprob, void* d_grad,
                                                      int32_t grad_type, int64_t ld_grad, float grad_scale, void* d_workspace,
                                                      int64_t workspace_bytes, void* hip_stream);

/* Measurement aids, not part of the method: read-only kernels that move the bytes the head moves and
 * compute nothing, to measure what one launch of that size and access pattern can reach on the chip.
 *   nanospec_calib_stream_read : reads d_buf[0, bytes) once, contiguously (bytes a multiple of 16).
 *   nanospec_calib_gather_read : reads the d bf16 of every row W[ids_b[j]], j < n_b, of sequence 0 of the
 *                                state's active list (the rows nanospec_sparse_head would gather).
 *   d_sink : device scratch of at least 1024 bytes (written practically never).
 *   nanospec_calib_valu_head   : the sparse head of one sequence (Eq. 1 on the active rows) computed on the
 *                                vector ALUs (unpack + fused multiply-add) instead of the matrix cores, with the
 *                                workgroup shape and loads of the product kernel for M <= 8: the measurement
 *                                behind the choice of the matrix cores below 16 hidden rows.  Logits as
 *                                nanospec_sparse_head (same layout and tolerance; the summation order differs).
 *                                batch == 1, M <= 8, d = 2048 or 4096, else EINVAL.
 * Errors: EINVAL (null, sizes < 1, bytes % 16 != 0).  Asynchronous. */
NANOSPEC_API nanospec_status nanospec_calib_valu_head(nanospec_state* st, const void* d_W_bf16, const void* d_H_bf16, int32_t M,
                                                      float* d_logits, void* hip_stream);
NANOSPEC_API nanospec_status nanospec_calib_stream_read(const void* d_buf, int64_t bytes, void* d_sink, void* hip_stream);
NANOSPEC_API nanospec_status nanospec_calib_gather_read(nanospec_state* st, const void* d_W_bf16, void* d_sink,
                                                        void* hip_stream);

/* Read and clear the sticky device error flags (NANOSPEC_DEV_* bits).  Synchronises `hip_stream`. */
NANOSPEC_API nanospec_status nanospec_last_device_error(nanospec_state* st, int32_t* flags, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* NANOSPEC_H_ */
