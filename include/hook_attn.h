/*
 * hook_attn.h -- C ABI of the hooked paged-attention library for NVIDIA B200 (sm_100a).
 *
 * One call computes, for a batch of sequences whose keys/values live in a paged KV cache,
 *
 *   (1) causal grouped-query attention   out[i,h,:] = softmax_t(scale * q[i,h,:].K[t,kv(h),:]) . V[t,kv(h),:]
 *   (2) the passive probe: for every *probed* query head and every configured key span
 *       [a_j, b_j) the exact post-softmax attention mass the query row places on the span,
 *           span_mass[i,h,j] = sum_{t in [a_j,b_j), t <= pos(i)} p[i,h,t]
 *       -- the quantity the paper's analyzer re-assembles from saved queries and keys and
 *       aggregates over token ranges (Section 2.2, the AttntrackerAnalyzer listing:
 *       "compute_attention_from_qk" followed by "attn2score" over "input_range"); the
 *       probed heads are the config's "important_heads" of one layer (Section 2, config
 *       listing), the probed rows its "hookq_mode" (last_token / all_tokens);
 *   (3) the active intervention: out[i,h,:] += alpha[h] * steer_vec[h,:] on the steered
 *       heads -- activation steering (Section 1, "Model Steering"; Section 3), applied per
 *       attention head after the softmax normalisation and before the single rounding of
 *       the output to bf16.
 *
 * Probing never changes `out` (Section 1 requires that passive programming leaves the model's
 * generation as it is): with and without probes the output bits are identical.  No attention matrix is materialised and no
 * query/key tensor leaves the GPU; span masses are carried as extra online-softmax
 * accumulators.
 *
 * Geometry.  Sequence s has L_s = seq_lens[s] keys in the cache (INCLUDING the keys of the
 * rows in this call: their K/V must already be written) and n_s query rows in this call.
 * Row i of sequence s sits at absolute position pos = L_s - n_s + i and sees keys 0..pos.
 * Logical key t of sequence s lives in physical page block_table[s][t / page_size], slot
 * t % page_size.  Query head h reads KV head h / (num_q_heads / num_kv_heads).
 *
 * Pointers.  Unless a field says "host", every pointer is a DEVICE pointer owned by the
 * caller and borrowed until the work enqueued by the call has completed on the stream.  The
 * attention calls write only `out`, `span_mass`, `workspace` and `status`.  Calls enqueue work on the
 * caller's stream, never synchronise, and never allocate device memory.  Return codes are
 * synchronous and cover argument validation and launch errors; faults the device detects
 * (a block-table entry outside [0, num_blocks), a sequence longer than its table, more rows
 * than keys, a sequence longer than `max_seq_len`) are reported through the optional `status`
 * word, the affected rows of `out` and `span_mass` are written as zeros, and no out-of-range
 * address is dereferenced.  Every entry point that launches work returns
 * HOOK_ATTN_ERR_INVALID_ARG unless the handle's device is the current device.
 *
 * Supported: head_dim in {64, 128}; page_size = 16; num_q_heads % num_kv_heads == 0 with a
 * group size <= 8; num_q_heads <= 64; num_spans <= 8; strides multiples of 8 elements and
 * 16-byte aligned base pointers.  Anything else returns HOOK_ATTN_ERR_UNSUPPORTED.
 */
#ifndef HOOK_ATTN_H_
#define HOOK_ATTN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hook_attn_handle hook_attn_handle; /* per-device state: SM count, cache of the prefill
                                                     kernel's TMA descriptors (keyed by pointer, shape, strides) */

enum {
    HOOK_ATTN_OK = 0,
    HOOK_ATTN_ERR_INVALID_ARG = -1, /* null required pointer, negative size, inconsistent shapes */
    HOOK_ATTN_ERR_UNSUPPORTED = -2, /* shape outside the supported set listed above */
    HOOK_ATTN_ERR_WORKSPACE = -3,   /* workspace missing or smaller than hook_attn_workspace_bytes */
    HOOK_ATTN_ERR_CUDA = -4,        /* a CUDA runtime/driver call failed (launch, attribute) */
    HOOK_ATTN_ERR_TIMEOUT = -5,     /* device status: a bounded wait inside a kernel ran out */
    HOOK_ATTN_ERR_BOUNDS = -6,      /* device status: block id / length outside its range */
    HOOK_ATTN_ERR_NO_PAGES = -7     /* device status: hook_cache_extend ran out of free pages */
};

/* Which query rows of a prefill call are probed: the config's "hookq_mode" (Section 2). */
enum {
    HOOK_PROBE_ROWS_ALL = 0,  /* "all_tokens": span_mass has one row per query row */
    HOOK_PROBE_ROWS_LAST = 1  /* "last_token": one row per sequence (its last query row) */
};

typedef struct {
    /* ---- shapes ---- */
    int32_t num_seqs;            /* sequences in the batch (>= 0) */
    int32_t total_q;             /* total query rows T = sum n_s (decode: == num_seqs) */
    int32_t num_q_heads;         /* Hq */
    int32_t num_kv_heads;        /* Hkv */
    int32_t head_dim;            /* D */
    int32_t page_size;           /* tokens per KV page */
    int32_t num_blocks;          /* physical pages in the cache (bounds for block_table) */
    int32_t max_blocks_per_seq;  /* row length of block_table */
    int32_t num_spans;           /* S spans per sequence (0 = no probe) */
    int32_t probe_rows;          /* HOOK_PROBE_ROWS_*; ignored by decode (always LAST) */
    float   scale;               /* softmax scale; <= 0 selects 1/sqrt(head_dim) */
    int32_t max_seq_len;         /* optional host-side bound on seq_lens (0 = unknown, then
                                    max_blocks_per_seq * page_size).  Block tables are often padded to
                                    the model's maximum length; with the bound, decode cuts its work and
                                    sizes its workspace for the lengths the batch really has.  A sequence
                                    longer than the bound is a device-detected fault (status, zeros). */

    /* ---- device tensors ---- */
    const void*    q;            /* bf16 [total_q][Hq][D], contiguous */
    const void*    k_cache;      /* bf16, element (block, slot, kv_head, d) at
                                    block*kv_block_stride + slot*kv_token_stride + kv_head*kv_head_stride + d */
    const void*    v_cache;      /* same layout and strides as k_cache */
    int64_t        kv_block_stride, kv_token_stride, kv_head_stride; /* in elements */
    const int32_t* block_table;  /* [num_seqs][max_blocks_per_seq]; entries past ceil(L_s/page_size)
                                    are never read */
    const int32_t* seq_lens;     /* [num_seqs] L_s */
    const int32_t* cu_q_lens;    /* [num_seqs+1] prefix sums of n_s; prefill only (decode: NULL) */
    const int32_t* spans;        /* [num_seqs][S][2] half-open absolute key ranges [a,b); clipped to the
                                    visible keys; a >= b is an empty span.  NULL = no probe */
    const float*   steer_vec;    /* fp32 [Hq][D]; NULL = no steering */
    void*          out;          /* bf16 [total_q][Hq][D] */
    float*         span_mass;    /* fp32 [rows][P][S]; rows = total_q (ALL) or num_seqs (LAST, decode);
                                    P = number of nonzero head_mask entries; the slot of a probed head is
                                    its rank among the probed heads in ascending head order.  In LAST mode
                                    a sequence without rows in the call gets zeros */
    void*          workspace;    /* scratch of at least hook_attn_workspace_bytes(); 256-byte aligned
                                    (checked: HOOK_ATTN_ERR_WORKSPACE otherwise) */
    size_t         workspace_bytes;
    int32_t*       status;       /* optional: one int32, set to a negative HOOK_ATTN_ERR_* code by the
                                    device on a detected fault; the caller zeroes it beforehand */

    /* ---- HOST arrays, read during the call and copied into the kernel parameters ---- */
    const uint8_t* head_mask;    /* host [Hq]; nonzero = probed head.  NULL = no probe */
    const float*   alpha;        /* host [Hq]; 0 = head not steered.  NULL = no steering */
} hook_attn_params;

/* Create / destroy the per-device handle.  `device` is a CUDA device ordinal.  Creation queries
 * device properties and configures the kernels; it fails with HOOK_ATTN_ERR_UNSUPPORTED on a
 * device that is not compute capability 10.x, HOOK_ATTN_ERR_CUDA if no device is usable. */
int hook_attn_create(hook_attn_handle** handle, int device);
int hook_attn_destroy(hook_attn_handle* handle);

/* Bytes of scratch the call described by `p` needs (only the shape fields and max_seq_len are read;
 * pass the same max_seq_len to the call).
 * is_decode = 1 sizes hook_attn_decode, 2 the decode half of hook_attn_mixed, 3 hook_attn_decode_q4, 0 hook_attn_prefill.
 * Returns 0 when the call needs no scratch or when the shapes are invalid. */
size_t hook_attn_workspace_bytes(const hook_attn_params* p, int is_decode);

/* Prefill / chunked prefill: n_s >= 0 rows per sequence given by cu_q_lens, n_s <= L_s.
 * (Section 2.2 recompute + Section 2 steering, fused into the attention forward.) */
int hook_attn_prefill(hook_attn_handle* handle, const hook_attn_params* p, void* cuda_stream);

/* Decode: exactly one query row per sequence (total_q == num_seqs, cu_q_lens ignored).  The keys of a
 * (sequence, KV head) unit are cut into pieces that are reduced independently and then merged.  The
 * cut is chosen from the host-known shape of the batch: with many units (num_seqs * num_kv_heads >=
 * 296) every sequence is cut into chunks of a fixed length (a power of two in 256..2048 keys, from
 * num_seqs, num_kv_heads and the length bound); with fewer, the pages of all units form one list
 * that is dealt out in equal shares to a fixed number of worker warps.  Either way the pieces of a
 * unit are merged in a fixed order, so results are bit-identical from run to run.  span_mass has one
 * row per sequence. */
int hook_attn_decode(hook_attn_handle* handle, const hook_attn_params* p, void* cuda_stream);

/* One step of a serving loop that holds both a decode batch and prefill chunks (chunked prefill, the
 * usual shape of a served step): the work of hook_attn_decode(decode) and hook_attn_prefill(prefill), same
 * arguments, outputs, results and error behaviour, issued together.  (Section 2: the hooks act inside the
 * engine's forward pass, whatever mix of requests a step carries; Section 2.1: the worker runs them per
 * execute_model call.)  When both halves have head_dim 128, the prefill half has at least 128 rows and the
 * decode half at most 512 sequences, one launch carries both -- a part of the SMs streams the decode batch
 * at HBM speed while the rest runs the prefill tiles on the tensor cores -- followed by the merge of the
 * decode partials; otherwise the two calls are issued one after the other.  `decode->workspace` must hold
 * hook_attn_workspace_bytes(decode, 2) bytes.  Either half may be empty (num_seqs = 0).  The two halves must
 * not write overlapping outputs. */
int hook_attn_mixed(hook_attn_handle* handle, const hook_attn_params* prefill, const hook_attn_params* decode,
                    void* cuda_stream);

/* Decode for callers that can neither allocate device memory nor hand over scratch.
 * (The paper has no counterpart; this is a convenience of the library.)
 *
 * Who needs it: code that runs where device allocation is off limits -- a serving loop whose
 * memory budget is already committed to the KV cache, a plug-in that only receives the hooked
 * layer's tensors, or a latency-critical path where an allocation (and the synchronisation it
 * implies) must never happen.  Such a caller cannot size and keep the `workspace` of
 * hook_attn_decode, so here the split-K partials go into a fixed array of
 * HOOK_ATTN_STATIC_SCRATCH_BYTES that is part of the library image: every GPU that loads the
 * library holds that much memory until the process exits.
 *
 * Same arguments, outputs and results as hook_attn_decode; `workspace` and `workspace_bytes` are
 * ignored.  The call allocates nothing and frees nothing.  A batch whose partials do not fit the
 * array (hook_attn_workspace_bytes(p, 1) > HOOK_ATTN_STATIC_SCRATCH_BYTES) is refused with
 * HOOK_ATTN_ERR_WORKSPACE and nothing is launched.  The handle's device must be the current
 * device, otherwise HOOK_ATTN_ERR_INVALID_ARG.
 *
 * The first call on each device looks up the device address of the array; make that first call
 * outside of any stream capture.  All calls on a device share the one array, which keeps whatever
 * the previous call left in it: the kernels never read an entry they have not written in the
 * same call, so nothing needs clearing -- but two calls whose work overlaps on the GPU (different
 * streams, or concurrent host threads) race on it.  Issue them on one stream, or order them. */
#define HOOK_ATTN_STATIC_SCRATCH_BYTES (16u << 20)
int hook_attn_decode_static_scratch(hook_attn_handle* handle, const hook_attn_params* p, void* cuda_stream);

/* Analyzer reduction over span masses (Section 2.2: the analyzer turns the re-assembled attention of
 * the important heads and the configured token ranges into a score, attn_func "sum_normalize";
 * Section 3: focus score of the instruction, per-passage relevance scores).  The analyzer's body is
 * not printed in the paper, so the two reductions are this library's reading of its words:
 *   HOOK_SCORE_MEAN            scores[r][j] = mean over probed heads p of span_mass[r][p][j]
 *   HOOK_SCORE_SUM_NORMALIZE   scores[r][j] = mean over p of span_mass[r][p][j] / sum_j' span_mass[r][p][j']
 *                              (a head whose masses sum to zero contributes zero); with the two spans
 *                              (instruction, data) scores[r][0] is instruction / (instruction + data).
 * span_mass: device fp32 [rows][num_probed][num_spans] as written by prefill / decode; scores: device
 * fp32 [rows][num_spans].  Only this small result has to leave the GPU. */
enum { HOOK_SCORE_MEAN = 0, HOOK_SCORE_SUM_NORMALIZE = 1 };
int hook_attn_score(hook_attn_handle* handle, const float* span_mass, int32_t rows, int32_t num_probed,
                    int32_t num_spans, int32_t mode, float* scores, void* cuda_stream);

/* Residual-stream activation steering (Section 1 "Model Steering", Section 3: a steering vector is
 * injected into a layer of the deployed model): hidden[t][:] += alpha * steer_vec[:] for every token
 * row t, in place.  hidden: device bf16, num_tokens rows of hidden_size elements, row_stride elements
 * apart (multiples of 8, 16-byte aligned); steer_vec: device fp32 [hidden_size].  The add is done in
 * fp32 and rounded once to bf16.  alpha = 0 changes nothing. */
int hook_steer_residual(hook_attn_handle* handle, void* hidden, const float* steer_vec, float alpha,
                        int64_t num_tokens, int32_t hidden_size, int64_t row_stride, void* cuda_stream);

/* Raw q/k capture (Section 2.1: the worker's hook keeps, per hooked attention module, the queries of the
 * last or of all tokens and the keys of all tokens; Section 2.2: the analyzer recomputes attention from
 * them).  For analyzers that need the raw states rather than span masses.  Reads q, k_cache, block_table,
 * seq_lens, cu_q_lens (prefill), head_mask (host) and probe_rows of `p`; spans, steering, out and
 * workspace are ignored.  With P probed heads in ascending order:
 *   q_out  device bf16 [rows][P][D], rows = total_q (all_tokens) or num_seqs (last_token / decode; a
 *          sequence without rows in the call gets zeros);               may be NULL
 *   k_out  device bf16 [sum L_s][P][D]: key t of sequence s at row cu_k_lens[s] + t, taken from the KV
 *          head of the probed query head;                               may be NULL
 *   cu_k_lens  device int32 [num_seqs + 1], prefix sums of seq_lens (caller-computed).
 * Byte-exact copies; block ids are bounds-checked like in the attention calls. */
int hook_capture_qk(hook_attn_handle* handle, const hook_attn_params* p, int is_decode, void* q_out, void* k_out,
                    const int32_t* cu_k_lens, void* cuda_stream);

/* Self-test of the kernels' bounded waits (the paper has no counterpart; it backs the failure
 * behaviour stated above).  Launches one small kernel that waits on a barrier nothing ever signals.
 * After `limit_ns` (1 .. 1e9) the wait gives up, the kernel writes HOOK_ATTN_ERR_TIMEOUT into the
 * device word `status` (zeroed by the caller), stores the time it waited into the optional device
 * word `waited_ns`, and returns normally: no trap, no hang, the context stays usable. */
int hook_attn_selftest_wait_limit(hook_attn_handle* handle, int32_t* status, uint64_t limit_ns, uint64_t* waited_ns,
                                  void* cuda_stream);

/* ---- what a decode step needs around the attention -------------------------------------------------------
 * (The paper leaves all of it to the engine it plugs into: Section 2.1, execute_model runs the model's forward
 * pass over the engine's cache.)  The conventions above hold: device pointers unless a field says host, the
 * caller's stream, no synchronisation, no allocation, HOOK_ATTN_ERR_INVALID_ARG unless the handle's device is
 * current, an optional status word for what only the device can see. */

enum { HOOK_DTYPE_BF16 = 0, HOOK_DTYPE_F16 = 1, HOOK_DTYPE_F32 = 2 };

/* Which axis turns which pair of a head: the pairs of axis 0, then those of axis 1, ... (BLOCKED), or dealt
 * out in turn, one to each axis that still has some left (CYCLIC). */
enum { HOOK_ROPE_AXES_BLOCKED = 0, HOOK_ROPE_AXES_CYCLIC = 1 };
/* Which elements of a head form pair p: p and p + rotary_dim / 2, or 2 p and 2 p + 1. */
enum { HOOK_ROPE_PAIR_HALVES = 0, HOOK_ROPE_PAIR_ADJACENT = 1 };
#define HOOK_ROPE_MAX_AXES 4

typedef struct {
    /* ---- shapes ---- */
    int32_t num_seqs, total_q, num_q_heads, num_kv_heads, head_dim, page_size, num_blocks, max_blocks_per_seq;
    int32_t dtype;               /* HOOK_DTYPE_* of q, k and v; what is written is bf16 */
    int32_t rotary_dim;          /* R, even, 0 .. head_dim: the first R elements of a head are rotated */
    int32_t num_axes;            /* 1 .. HOOK_ROPE_MAX_AXES (time, height, width, ...) */
    int32_t axis_pairs[HOOK_ROPE_MAX_AXES]; /* pairs of each axis; they add up to R / 2 */
    int32_t axis_order;          /* HOOK_ROPE_AXES_* */
    int32_t pairing;             /* HOOK_ROPE_PAIR_* */
    float   factor;              /* multiplies cosines and sines (long-context scalings); finite, 0 selects 1 */

    /* ---- device tensors ---- */
    const void*    q;            /* [total_q][Hq][D], strides in elements; the last one is 1 */
    const void*    k;            /* [total_q][Hkv][D] */
    const void*    v;            /* [total_q][Hkv][D] */
    int64_t        q_row_stride, q_head_stride, k_row_stride, k_head_stride, v_row_stride, v_head_stride;
    const float*   inv_freq;     /* fp32 [R / 2]; NULL when R = 0 */
    const int32_t* positions;    /* [num_axes][total_q], axes position_axis_stride apart; NULL: every axis has the
                                    row's position in its sequence */
    int64_t        position_axis_stride;
    void*          q_out;        /* bf16 [total_q][Hq][D], contiguous; may be q itself (bf16 and contiguous), and
                                    overlaps none of the inputs otherwise */
    void*          k_cache;      /* as in hook_attn_params, written here */
    void*          v_cache;
    int64_t        kv_block_stride, kv_token_stride, kv_head_stride;
    const int32_t* block_table;
    const int32_t* seq_lens;     /* L_s INCLUDING this call's rows */
    const int32_t* cu_q_lens;    /* [num_seqs + 1]; NULL: decode, one row per sequence, total_q == num_seqs */
    int32_t*       status;
} hook_rope_params;

/* Rotary positions with several axes, appended to the cache: what the rows of a call need before
 * hook_attn_prefill / hook_attn_decode.  Pair p of a q or k head turns by positions[axis(p)][row] * inv_freq[p]:
 *   (a, b) -> factor * (a cos - b sin, b cos + a sin)
 * with the angle reduced in 64 bits, the rest in 32, and one rounding to bf16.  k and v of row i of sequence s go
 * to position L_s - n_s + i of its pages; the pages that are written belong to one sequence alone
 * (hook_cache_extend sees to it).  Rows behind cu_q_lens[num_seqs] are left as they were.  A row whose sequence
 * or page is out of range (L_s beyond its table, n_s > L_s, a block id outside the pool) sets status, its q_out
 * row is zeroed and nothing is appended for it. */
int hook_rope_append(hook_attn_handle* handle, const hook_rope_params* p, void* cuda_stream);

typedef struct {
    int32_t num_rows, vocab_size, max_tokens, num_bias, num_masks;
    int32_t dtype, out_dtype;    /* HOOK_DTYPE_* of logits; of out: the same, or HOOK_DTYPE_F32 */
    const void*     logits;      /* [num_rows][vocab_size], rows logits_row_stride elements apart */
    void*           out;         /* may be logits itself (same type and stride), and overlaps nothing otherwise */
    int64_t         logits_row_stride, out_row_stride;
    const int32_t*  tokens;      /* [num_rows][max_tokens]: a row's prompt, then what was generated; ids outside
                                    [0, vocab_size) (placeholders) are passed over.  NULL: no penalties */
    int64_t         tokens_row_stride; /* 0: all rows have the same */
    const int32_t*  prompt_lens; /* [num_rows] tokens of the prompt */
    const int32_t*  total_lens;  /* [num_rows] tokens of prompt and generation, prompt_lens <= total_lens <= max_tokens */
    const float*    repetition;  /* [num_rows], > 0; NULL: 1 */
    const float*    presence;    /* [num_rows]; NULL: 0 */
    const float*    frequency;   /* [num_rows]; NULL: 0 */
    const int32_t*  bias_offsets;/* [num_rows + 1] prefix sums of the rows' bias entries, at most 2047 a row;
                                    NULL: no biases */
    const int32_t*  bias_tokens; /* [num_bias]; of a token named twice in a row the last entry counts */
    const float*    bias_values; /* [num_bias] */
    const uint32_t* mask;        /* [num_masks][ceil(vocab_size / 32)], bit v % 32 of word v / 32: token v is
                                    allowed.  NULL: no grammar */
    int64_t         mask_row_stride; /* in words; 0: all masks are the same */
    const int32_t*  mask_rows;   /* [num_rows] row of mask, negative: the row has no grammar.  NULL: row r has mask r */
    int32_t*        status;
} hook_logits_params;

/* Edits of the logits before a token is chosen, in 32 bits with one rounding to out's type.  With c the number of
 * times token v was generated in the row, and `seen` whether it is in its prompt or generated:
 *   x = seen ? (x > 0 ? x / repetition : x * repetition) : x;   x -= frequency * c + presence  if c > 0 (either may be infinite);
 *   x += bias[v];   x = -inf if the grammar forbids v (whatever x is; a mask may forbid all).
 * A row whose lengths, bias offsets or mask row are out of range sets status and its part of out is not written; a
 * bias for a token outside the vocabulary sets status and is passed over.  vocab_size <= 2^20, max_tokens < 2^20, num_rows < 2^16. */
int hook_adjust_logits(hook_attn_handle* handle, const hook_logits_params* p, void* cuda_stream);

/* The pool that the sequences of a cache share.  All its arrays are written by the calls below. */
typedef struct {
    int32_t  num_seqs, max_blocks_per_seq, num_blocks, page_size;   /* num_seqs <= 16384, at most 2^30 pages and 2^30 entries */
    int32_t* block_table;        /* [num_seqs][max_blocks_per_seq] */
    int32_t* seq_lens;           /* [num_seqs] tokens; 0: the row is empty */
    int32_t* page_refs;          /* [num_blocks] sequences that hold the page; 0 (or less): free */
    int32_t* status;
} hook_cache_pool;

/* children[i] becomes a copy of sequence parents[i] that shares its pages (no data moves).  An entry is passed
 * over, with status HOOK_ATTN_ERR_BOUNDS, when one of its rows does not exist, its child is not empty, is named by
 * an earlier entry or is a parent in this call, or the parent's length or pages are out of range or nobody holds one of
 * its pages.  At most 16384 entries, here and in hook_cache_free. */
int hook_cache_fork(hook_attn_handle* handle, const hook_cache_pool* pool, const int32_t* parents, const int32_t* children,
                    int32_t num_forks, void* cuda_stream);

/* Room for new_rows[s] >= 0 more tokens in every sequence: the missing pages are taken from the pool, lowest ids
 * first and in the order of the sequences, and seq_lens grows.  A sequence that would write into a partly filled
 * page that it shares gets a page of its own instead, and pairs[s] = (old page, new page) for
 * hook_cache_copy_pages; else pairs[s] = (-1, -1).  Copy the pairs before anything is appended and before the next
 * call here: a page that all its sharers leave in one call is free afterwards.  Sequences that the pool cannot serve in their turn stay as
 * they are and set status HOOK_ATTN_ERR_NO_PAGES; those whose length, table or last page is out of range stay as
 * they are and set HOOK_ATTN_ERR_BOUNDS.  pairs: int32 [num_seqs][2]. */
int hook_cache_extend(hook_attn_handle* handle, const hook_cache_pool* pool, const int32_t* new_rows, int32_t* pairs,
                      void* cuda_stream);

/* Cuts sequence seqs[i] to its first keep_lens[i] tokens (NULL: 0, the whole sequence goes; more than it has:
 * nothing happens): the pages behind them are given back, or to the others that share them, and their table
 * entries become -1.  Of a sequence that is named twice the first entry counts.  A row that does not exist, a
 * negative or too long length and a page that nobody holds set status. */
int hook_cache_free(hook_attn_handle* handle, const hook_cache_pool* pool, const int32_t* seqs, const int32_t* keep_lens,
                    int32_t num_entries, void* cuda_stream);

/* Plans how the U pages in use move together at the low end of the pool: the k-th used page at U or above goes to
 * the k-th free page below U.  The pool itself is only read, so that the old tables stay valid until the pairs are
 * copied.  Outputs: block_table_out (like block_table; may be block_table itself; -1 behind a sequence's pages),
 * page_refs_out (like page_refs; neither it nor page_map is page_refs itself), page_map int32 [num_blocks] (where each page is afterwards,
 * -1: free), pairs int32 [num_blocks / 2][2] (source, destination; -1 behind the last), num_pairs int32 [1]. */
int hook_cache_compact(hook_attn_handle* handle, const hook_cache_pool* pool, int32_t* block_table_out, int32_t* page_refs_out,
                       int32_t* page_map, int32_t* pairs, int32_t* num_pairs, void* cuda_stream);

typedef struct {
    int32_t num_layers, num_blocks, page_size, num_kv_heads, head_dim, max_pairs;
    int64_t kv_block_stride, kv_token_stride, kv_head_stride;   /* of every layer's caches, in elements */
    void* const*   k_caches;     /* HOST array [num_layers] of device pointers */
    void* const*   v_caches;     /* HOST array [num_layers] */
    const int32_t* pairs;        /* [max_pairs][2] source and destination page; a negative one: passed over; max_pairs <= 2^30 */
    const int32_t* num_pairs;    /* device int32 [1], how many of them count; NULL: max_pairs */
    int32_t*       status;
} hook_cache_copy_params;

/* Copies pages in the caches of all layers.  A source may have many destinations.  The pairs are independent of one
 * another: one whose destination is also another pair's destination or source, or whose source is another pair's
 * destination, is not carried out and sets status, like one outside the pool.  They are held against one another, which takes a time that
 * grows with the square of their number (2^18 pairs: 30 ms): of more than 2^22 that count, none is carried out and status is set. */
int hook_cache_copy_pages(hook_attn_handle* handle, const hook_cache_copy_params* p, void* cuda_stream);

/* ---- a cache held in 4 bits ----------------------------------------------------------------------------------
 * Where the cache and not the model bounds the number of sequences: keys and values of 16 tokens in 2.1 to 2.5 KB a
 * head of 128 instead of 8 KB.  Block tables, lengths and the pool calls above are as for a bf16 cache; the pages are
 * written by hook_rope_append_q4, read by hook_attn_decode_q4, and read back to bf16 pages for whatever else reads a
 * cache (hook_attn_prefill of a prompt's next chunk, hook_capture_qk) by hook_cache_read_q4.  A sequence has at most 2^31 - 4096 tokens; a longer
 * one is a fault, like one that is longer than its table.
 *
 * A head's elements share a step and a lowest value in groups of `group` neighbours.  Of the group's elements, rounded
 * to bf16 (what a bf16 cache holds), lowest is the least, step = (greatest - lowest) / 15, both in 32 bits, rounded to bf16 (0 if
 * that is below 2^-100), and an element x has the code nearest to (x - lowest) / step, 0 .. 15, x - lowest rounded to 32 bits and halves
 * to even (0 where the step is 0).  It reads as lowest + step * code.  A group that holds an infinity or a NaN, or whose greatest - lowest
 * overflows 32 bits, reads as NaN.
 *
 * A page's part for one KV head is a slab of hook_q4_slab_bytes(head_dim, group) bytes: 16 head_dim / 2 bytes of K codes, as
 * many of V codes, then for K and for V the pairs (step, lowest) of bf16 [16][head_dim / group].  The codes of token t, element e:
 *   K  nibble e % 8 (of a little-endian 32-bit word) of word (e / 8 % 4) * (head_dim / 32) + e / 32 of row t;
 *   V  nibble e % 32 / 8 of the 16-bit word e / 32 of unit u of row (t / 2 % 4) + 4 (t % 2) + 8 (t / 8), a unit having head_dim / 16 bytes and
 *      u being e % 8, with head_dim 128 and a row whose bit 1 is set e % 8 xor 4. */
typedef struct {
    void*   pages;               /* slab of block b, KV head h at b * block_stride + h * head_stride; 16-byte aligned */
    int64_t block_stride, head_stride;  /* in BYTES, multiples of 16 */
    int32_t group;               /* elements to a group: 32, 64 or 128, at most head_dim */
} hook_q4_cache;

/* Bytes of a slab; 0 for a head_dim or group that is not supported. */
size_t hook_q4_slab_bytes(int32_t head_dim, int32_t group);

/* hook_rope_append into a 4-bit cache: the same queries, keys rotated and rounded to bf16 in the same way, then keys and values
 * quantised as they are written.  k_cache, v_cache and the kv strides of `p` are ignored; q_out must not overlap the pages. */
int hook_rope_append_q4(hook_attn_handle* handle, const hook_rope_params* p, const hook_q4_cache* cache, void* cuda_stream);

/* hook_attn_decode over a 4-bit cache: the same arguments, outputs, hooks and faults, k_cache, v_cache and the kv strides of `p` being
 * ignored.  `workspace` holds hook_attn_workspace_bytes(p, 3) bytes.  Scores, softmax, span masses and the sums over the values
 * are in 32 bits; a probability times a step of V is rounded to 11 bits or, below 2^-20 of the largest probability times the largest step of
 * the same group, to within 2^-31 of the latter.  Elements of q below 2^-27 of their head's largest are rounded to within 2^-35 of it. */
int hook_attn_decode_q4(hook_attn_handle* handle, const hook_attn_params* p, const hook_q4_cache* cache, void* cuda_stream);

typedef struct {
    int32_t num_seqs, num_kv_heads, head_dim, page_size;
    int32_t num_blocks, max_blocks_per_seq;         /* of the 4-bit cache and its block_table */
    int32_t to_num_blocks, to_max_blocks_per_seq;   /* of the bf16 cache and to_table */
    const int32_t* block_table;  /* [num_seqs][max_blocks_per_seq] */
    const int32_t* seq_lens;     /* [num_seqs]; 0: nothing is read */
    const int32_t* first;        /* [num_seqs] first position that is read; NULL: 0 */
    void*          k_cache;      /* bf16, written: as in hook_attn_params */
    void*          v_cache;
    int64_t        kv_block_stride, kv_token_stride, kv_head_stride;
    const int32_t* to_table;     /* [num_seqs][to_max_blocks_per_seq] pages of the bf16 cache */
    int32_t*       status;
} hook_q4_read_params;

/* Positions first[s] .. seq_lens[s] - 1 of every sequence, each lowest + step * code computed in 32 bits and rounded to bf16, go to the
 * same positions of to_table's pages; nothing else is written.  The pages that are written belong to one sequence
 * alone.  A sequence whose length is negative or beyond one of the tables, or whose first is negative, is passed over and sets status, like
 * a page outside its pool. */
int hook_cache_read_q4(hook_attn_handle* handle, const hook_q4_read_params* p, const hook_q4_cache* cache, void* cuda_stream);

typedef struct {
    int32_t num_layers, num_blocks, page_size, num_kv_heads, head_dim, group, max_pairs;
    int64_t block_stride, head_stride;   /* of every layer's pages, in bytes */
    void* const*   pages;        /* HOST array [num_layers] of device pointers */
    const int32_t* pairs;        /* as in hook_cache_copy_params */
    const int32_t* num_pairs;
    int32_t*       status;
} hook_q4_copy_params;

/* hook_cache_copy_pages for 4-bit caches. */
int hook_cache_copy_pages_q4(hook_attn_handle* handle, const hook_q4_copy_params* p, void* cuda_stream);

/* ---- the choice of a token ------------------------------------------------------------------------------------ */
typedef struct {
    int32_t num_rows, vocab_size;
    int32_t dtype;               /* HOOK_DTYPE_* of logits */
    const void*    logits;       /* [num_rows][vocab_size], rows logits_row_stride elements apart */
    int64_t        logits_row_stride;
    const float*   uniform;      /* [num_rows] random numbers in [0, 1) */
    const float*   temperature;  /* [num_rows] T >= 0; 0: the token with the largest logit; NULL: 1 */
    const int32_t* top_k;        /* [num_rows]; 0 or less, or vocab_size and more: all; NULL: all */
    const float*   top_p;        /* [num_rows] >= 0; 1 and more: all; NULL: all */
    const float*   min_p;        /* [num_rows] 0 .. 1; NULL: 0 */
    int32_t*       tokens;       /* [num_rows] */
    int32_t*       status;
} hook_sample_params;

/* One token for every row, from its logits (of hook_adjust_logits, say) and one random number.  Token v weighs w_v = exp((x_v - max x) / T).  In the
 * order of falling logits, equal ones in that of their indices, the first top_k tokens stay, of these those with
 * w_v >= min_p, and of these each before which less than top_p of their weight lies; the first one always stays.  The token is the first, in the
 * order of the indices, up to and with which the weights of those that stayed exceed `uniform` times their sum.
 * The weights are computed in 64 bits and summed as whole multiples of 2^-42: the order of the sums has no say in the result, and a
 * token below 2^-43 of the most likely one is never drawn.  Logits are taken to within 2^-126.  A NaN counts as -infinity; infinite logits weigh
 * the same, and the others nothing next to them.
 * A row without a logit above -infinity, or with a parameter outside the ranges above (NaN among them), gets -1 and sets status to
 * HOOK_ATTN_ERR_INVALID_ARG.  vocab_size <= 2^20, num_rows < 2^16. */
int hook_sample_tokens(hook_attn_handle* handle, const hook_sample_params* p, void* cuda_stream);

/* Human-readable name of a return / status code. */
const char* hook_attn_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* HOOK_ATTN_H_ */
