/*
 * td.h - C ABI of the transfer dock: put/get dispatch of RL samples held in GPU memory.
 *
 * The dock follows the sample flow of "Distributed Transfer Dock Strategy" (Fig. 4, Eq. 4):
 *   warehouses  hold the real data, the buffer being split along the global batch with every
 *               sample keeping its own index        -> per-column ragged arenas, S shards;
 *   controllers (one per worker state) record which samples that state may still be served
 *                                                   -> per-consumer claim / consumed bitmaps;
 *   workflow    1. a worker state asks its controller for metadata     (td_get: select)
 *               2. it fetches, or sends, the real data                 (td_get: gather, td_put)
 *               3. the warehouse updates its state, visible to every controller
 *                                                                      (td_put: publish).
 * The record schema is the one under Eq. 1: one prompt-length item, several response-length
 * items and a few scalars per sample; samples come in GRPO groups of N responses per prompt
 * (Fig. 2).  The group-normalised advantage is not given in the paper; td_get computes
 * A = (r - mean) / (std + eps) over each dispatched group, population std, in double.
 *
 * Conventions for every call:
 *   - "device" pointers are CUDA device memory owned by the caller; the library allocates no
 *     device memory and frees none.  "host" pointers are ordinary host memory.  The one
 *     allocation the library makes is pinned HOST memory: td_get_many_host with a staging
 *     buffer allocates a host mirror of it once per plan (freed by td_plan_destroy).
 *   - td_put / td_get / td_get_many / td_reset only enqueue work on the given stream and return;
 *     they never synchronise.  Calls on one stream execute in call order.  Gets may run
 *     concurrently with each other and with puts on other streams.  Puts that may reserve the
 *     same row (the first columns of a length class to arrive for a sample) must be ordered by
 *     the caller; puts of further columns for samples whose rows of that class are stored and
 *     published (the write-backs of worker states) only read the tables and may overlap.
 *   - return value: TD_OK (0) or a negative td_error found on the host.  Conditions found on the
 *     device never trap: the offending sample is skipped, a TD_ERR_* bit is OR-ed into the
 *     dock's error word (td_status) and, for a get, into td_result.status.
 *   - a streamlike argument is a cudaStream_t passed as void* (NULL = the default stream).
 */
#ifndef TD_H
#define TD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct td_dock td_dock;          /* opaque host object */

enum { TD_I32 = 0, TD_F32 = 1, TD_BF16 = 2 };             /* td_column.dtype */
enum { TD_SCALAR = 0, TD_PROMPT = 1, TD_RESPONSE = 2 };   /* td_column.cls   */
enum { TD_PACKED = 0, TD_PADDED = 1 };                    /* td_get_out.mode */
enum { TD_OUT_LEFT_PAD_PROMPT = 1u };                     /* td_get_out.flags */
enum { TD_F_ADVANTAGE = 1u };                             /* td_consumer.flags */

typedef enum {
    TD_OK = 0,
    TD_EINVAL = -1,       /* bad argument                                   */
    TD_EWORKSPACE = -2,   /* workspace or scratch too small or misaligned   */
    TD_ECUDA = -3,        /* a CUDA runtime call failed (no device, ...)    */
    TD_ETOOLARGE = -4     /* td_get_static: the dock exceeds its fixed scratch */
} td_error;

/* device-detected conditions */
enum {
    TD_ERR_OOB_INDEX        = 1u << 0,  /* put: sample index outside [0, G*N)                  */
    TD_ERR_DUP_PUT          = 1u << 1,  /* put: (sample, column) already stored; first one kept */
    TD_ERR_LEN_MISMATCH     = 1u << 2,  /* put: length differs from the sample's length class   */
    TD_ERR_ARENA_FULL       = 1u << 3,  /* put: shard arena has no room for the row             */
    TD_ERR_OUT_TRUNCATED    = 1u << 4,  /* get: stopped before a group that would not fit       */
    TD_ERR_LOOKBACK_TIMEOUT = 1u << 5,  /* get: a scan tile gave up waiting; nothing is served,
                                           nothing stays claimed, the groups remain available   */
    TD_ERR_BAD_LENGTH       = 1u << 6,  /* put: cu not monotone or beyond data_elems            */
    TD_ERR_COPY_TIMEOUT     = 1u << 7   /* a staged copy did not land in time; plain loads used.
                                           td_cache_attention: products did not come in time, see there */
};

typedef struct {
    const char *name;      /* not kept */
    int32_t  dtype;        /* TD_I32 | TD_F32 | TD_BF16; payload is copied as raw bits */
    int32_t  cls;          /* TD_SCALAR: one element per sample; TD_PROMPT / TD_RESPONSE:
                              a row whose length is the sample's prompt / response length */
    uint32_t pad_bits;     /* raw bit pattern written behind a row in TD_PADDED mode */
} td_column;

typedef struct {
    const char *name;      /* not kept */
    uint32_t need_mask;    /* bit c: column c must be stored before a sample is served */
    uint32_t out_mask;     /* bit c: column c is gathered; must lie within need_mask   */
    uint32_t flags;        /* TD_F_ADVANTAGE: needs reward_column within need_mask     */
} td_consumer;

typedef struct {
    uint32_t n_prompts;    /* G */
    uint32_t n_per_group;  /* N; sample s = prompt * N + response, group = s / N; G * N < 2^30 */
    uint32_t n_shards;     /* S warehouses, 1..256, must divide G; shard(s) = (s / N) / (G / S) */
    uint32_t n_columns;    const td_column   *columns;     /* 1..32, host array */
    uint32_t n_consumers;  const td_consumer *consumers;   /* 1..32, host array */
    uint64_t prompt_elems_per_shard;    /* arena capacity per shard, elements (rounded up to 8) */
    uint64_t response_elems_per_shard;
    uint32_t reward_column;             /* a TD_F32 TD_SCALAR column */
    float    adv_eps;
    int32_t  device;                    /* CUDA device ordinal of the workspace */
} td_config;

/* Written by td_get on the device; read it after the stream has reached that point. */
typedef struct {
    uint32_t n_samples, n_groups;             /* n_samples = n_groups * N */
    uint64_t prompt_tokens, response_tokens;  /* = cu_prompt[n_samples], cu_response[n_samples] */
    uint32_t status;                          /* TD_ERR_* bits of this call */
    uint32_t reserved;
} td_result;

/* Output buffers of one get.  The struct itself is host memory; every pointer in it is
 * caller-owned DEVICE memory that stays valid until the get has executed.  The payload buffers
 * (col[], seq, seq_advantages) may instead be page-locked host memory that the device can
 * address (cudaHostAlloc / cudaHostRegister under unified addressing): the gather then writes
 * the batch across the bus itself, in wide contiguous stores, and a worker whose tensors live on
 * the host needs no copy afterwards.  indices, the cu arrays, advantages and result are read
 * back by the kernels and belong in device memory. */
typedef struct {
    int32_t  mode;                    /* TD_PACKED: column c holds its rows back to back, row i at
                                         cu_<class>[i]; TD_PADDED: row i at i * pad_<class>_to,
                                         filled up with the column's pad_bits */
    uint32_t pad_prompt_to, pad_response_to;   /* row widths in elements (TD_PADDED only) */
    uint32_t flags;                   /* 0, or TD_OUT_LEFT_PAD_PROMPT: in TD_PADDED mode a row of a
                                         TD_PROMPT column ends at its width, (pad_prompt_to - length)
                                         copies of pad_bits in front of it, so that in a dense
                                         [prompt | response] batch every response starts at the same
                                         position, as batched generation lays its sequences out;
                                         TD_RESPONSE rows are padded behind as always, TD_PACKED
                                         ignores the flag.  Any other bit: TD_EINVAL */
    int32_t *indices;                 /* [max_samples] sample indices, ascending          required */
    int32_t *cu_prompt, *cu_response; /* [max_samples + 1] prefix sums of the true lengths required */
    int32_t *cu_seq;                  /* [max_samples + 1] cu_prompt + cu_response, or NULL */
    void    *col[32];                 /* per column; NULL = not wanted                     */
    uint64_t col_capacity_elems[32];  /* room behind col[c], in elements                   */
    float   *advantages;              /* [max_samples]; required iff TD_F_ADVANTAGE        */
    td_result *result;                /* required                                          */
    void    *scratch;                 /* td_get_scratch_bytes() bytes, 16-byte aligned, private to
                                         this call while it is in flight; zero-filled once after
                                         allocation, never needs clearing afterwards       required */
    uint64_t scratch_bytes;
    /* Fused token stream, optional (seq == NULL and seq_advantages == NULL: not wanted; a zeroed
     * struct asks for neither).  What a varlen trainer reads directly: sample i's row of column
     * seq_prompt_col (TD_PROMPT) followed by its row of column seq_response_col (TD_RESPONSE, same
     * element size, both within the consumer's out_mask) at element cu_seq[i] of `seq`, in
     * either output mode; cu_seq is then required.  seq_advantages (needs TD_F_ADVANTAGE) has the
     * same layout in float: 0 on prompt tokens, the sample's advantage on its response tokens,
     * i.e. advantage times loss mask.  seq_capacity_elems is the room behind each of the two; a
     * group that would not fit ends the batch (TD_ERR_OUT_TRUNCATED). */
    uint32_t seq_prompt_col, seq_response_col;
    void    *seq;
    uint64_t seq_capacity_elems;
    float   *seq_advantages;
} td_get_out;

typedef struct {
    uint64_t put_accepted[32];        /* per column */
    uint64_t got_samples[32];         /* per consumer */
    uint64_t got_tokens[32];          /* per consumer, prompt + response tokens */
    uint64_t n_oob, n_dup, n_len_mismatch, n_arena_full, n_truncated, n_bad_length;
    uint64_t n_claim_conflicts;       /* groups lost to a concurrent get of the same consumer */
    uint64_t n_lookback_timeouts;
    uint32_t error_word;              /* OR of all TD_ERR_* bits since the last reset */
    uint32_t reserved;
} td_stats;

/* Bytes of device workspace a dock with this configuration needs (tables, bitmaps and the
 * arenas of Eq. 4's payload term).  Host only; no CUDA call. */
int td_query_workspace(const td_config *cfg, size_t *bytes);

/* Builds a dock inside `d_workspace` (device, 256-byte aligned, `bytes` >= td_query_workspace)
 * and brings it to the empty state on the default stream, synchronising once.  The workspace
 * stays the caller's and must outlive the dock.  *out is freed by td_destroy. */
int td_create(const td_config *cfg, void *d_workspace, size_t bytes, td_dock **out);
int td_destroy(td_dock *dock);

/* Workflow steps 2 and 3 for a producer: store column `column` of the k samples d_indices[0..k)
 * and make them visible to every consumer.
 *   d_indices  device int32 [k], any order.
 *   d_cu       device int32 [k + 1], non-decreasing element offsets of the rows inside d_data;
 *              NULL for a TD_SCALAR column (row i is element i).
 *   d_data     device, rows back to back, data_elems elements in total (bounds what is read).
 * Rows are placed in call order: the first column of a length class to arrive for a sample
 * fixes its length and reserves its row at the next free element of the sample's shard.
 * Samples that are out of range, already stored, of the wrong length or without room are
 * skipped and counted.  The same index twice within one call is safe but leaves that row's
 * content unspecified. */
int td_put(td_dock *dock, uint32_t column, const int32_t *d_indices, uint32_t k,
           const int32_t *d_cu, const void *d_data, uint64_t data_elems, void *stream);

/* Workflow steps 1 and 2 for worker state `consumer`: claim the lowest-numbered groups whose
 * need_mask columns are all stored and that this consumer has not been served, at most
 * max_samples / N of them, and gather their out_mask columns, cu_seqlens and (TD_F_ADVANTAGE)
 * advantages into `out`.  Fewer groups than asked for, zero included, is not an error.  The
 * batch ends before the first group that would overflow a supplied buffer (TD_ERR_OUT_TRUNCATED;
 * that group stays available).  A group is never served twice to one consumer, also when gets
 * of that consumer run concurrently on several streams; such a get may then return fewer
 * groups than were ready. */
int td_get(td_dock *dock, uint32_t consumer, uint32_t max_samples, const td_get_out *out,
           void *stream);
size_t td_get_scratch_bytes(const td_dock *dock);

/* td_get for callers that cannot provide scratch memory.  (The paper has no counterpart: this
 * is a convenience of this library.)  Some code that wants to serve a batch may not allocate
 * device memory at all: a step running inside a serving loop whose memory pool is frozen, a
 * plug-in that is handed nothing but its input and output buffers, a process whose memory
 * budget is already committed.  td_get asks such a caller for td_get_scratch_bytes() of
 * zero-filled device memory it does not have.  td_get_static does the same get with the scan
 * scratch kept in a fixed array inside the library (about 65 KB, held by every GPU that loads
 * the library until the process exits); out->scratch and out->scratch_bytes are ignored, every
 * other field of `out` means what it means for td_get, and the results are the same.
 *   - Limit: docks of at most 16384 prompts (G); a larger dock gets TD_ETOOLARGE and nothing
 *     is enqueued.
 *   - The call allocates and frees nothing.  Its first call on a device looks the array's device
 *     address up (once per device; a host-side query, no allocation); make that first call
 *     outside any stream capture.
 *   - All calls share the one array, which still holds the previous call's contents; the words
 *     that must start at zero are cleared on `stream` before the scan.  Two td_get_static calls
 *     that overlap on the GPU (different streams, no ordering between them) race on it: they
 *     share the scan's ticket, its tile descriptors and its candidate list, so the outcome is
 *     undefined within the dock's own tables: either call may return nothing, report
 *     TD_ERR_LOOKBACK_TIMEOUT, be served groups that the other call selected (also groups of
 *     the other call's consumer, whose served marks are then set for the wrong worker state),
 *     or leave groups claimed and unserved until td_reset.  No memory outside the dock, the
 *     array and the two calls' own output buffers is touched.  Order such calls (one stream,
 *     or events), or use td_get with separate scratch for gets that may overlap. */
int td_get_static(td_dock *dock, uint32_t consumer, uint32_t max_samples, const td_get_out *out,
                  void *stream);

/* Several columns in one call, as a worker that sends a whole record does (prompt and response
 * ids together, say): the items are stored as if td_put had been called on each in array order,
 * with three kernel launches for up to eight items instead of three per item.  Every field of
 * an item means what the td_put argument of the same name means. */
typedef struct {
    uint32_t column, k;
    const int32_t *d_indices;
    const int32_t *d_cu;
    const void *d_data;
    uint64_t data_elems;
} td_put_item;
int td_put_many(td_dock *dock, const td_put_item *items, uint32_t n_items, void *stream);

/* Workflow steps 2 and 3 for a worker state that sends back what it computed from a batch it was
 * just served (the reference model's log-probs, the reward, ...), which is how readiness cascades
 * from generation through the inference states to the actor update (Fig. 1, Fig. 2): the samples
 * are the ones the get returned, and their number is read from the get's result block on the
 * device when the put executes, so the host neither waits for the get nor learns its size.
 *   batch        the td_get_out of that get (host struct, device pointers): indices, cu_prompt,
 *                cu_response and result are used and must stay valid until the put has executed;
 *                the put must be ordered behind the get (same stream, or an event).
 *   max_samples  upper bound of the batch size (the value given to the get).
 *   items        host array; column `column` takes row i of the batch from d_data (device) at
 *                element cu_<class>[i], i.e. rows packed in batch order exactly as a packed get
 *                lays them out; a TD_SCALAR column takes element i.  data_elems bounds what is
 *                read.
 * Everything else is td_put_many's: rows are placed and checked the same way, and the same
 * conditions are counted. */
typedef struct {
    uint32_t column, reserved;
    const void *d_data;
    uint64_t data_elems;
} td_back_item;
int td_put_back(td_dock *dock, const td_get_out *batch, uint32_t max_samples, const td_back_item *items,
                uint32_t n_items, void *stream);

/* The write-backs of several worker states in one call (three kernel launches for up to eight
 * of them): request r sends column `column` back for the batch `batch` it names, exactly as
 * td_put_back(dock, batch, max_samples, {column, d_data, data_elems}, 1, stream) would; the
 * requests are stored in array order.  Together with td_get_many this serves one poll of every
 * worker state with five or six launches, whatever their number. */
typedef struct {
    const td_get_out *batch;
    uint32_t max_samples, column;
    const void *d_data;
    uint64_t data_elems;
} td_back_req;
int td_put_back_many(td_dock *dock, const td_back_req *reqs, uint32_t n_reqs, void *stream);

/* Many gets served by one call.  Each worker state has its own controller and a step serves
 * several of them, each in several micro-batches; a plan fixes the list of requests (consumer,
 * max_samples, output buffers) once and td_get_many then serves all of them with three kernel
 * launches (two when the dock has at most 1024 prompts and every consumer one request).  Requests that name the same consumer are served in array order: the result is the
 * one td_get would give when called on each request in turn, except that a group cut off by
 * TD_ERR_OUT_TRUNCATED is not offered to the later requests of the same call.
 *   td_plan_bytes   device bytes a plan of n_req requests needs (request table + scan scratch).
 *   td_plan_create  checks the requests (host array; out.scratch is not used), uploads them into
 *                   d_plan (device, 256-byte aligned, caller-owned, must outlive the plan) on
 *                   `stream`.  n_req * n_columns must not exceed 4096, and the requests' output
 *                   room together must stay below 256 GiB (TD_EINVAL).
 *   td_get_many     enqueues the gets.  A plan must not be in flight twice at the same time;
 *                   reusing it on one stream, call after call, is the intended use. */
typedef struct {
    uint32_t consumer, max_samples;
    td_get_out out;
} td_get_req;
typedef struct td_plan td_plan;
size_t td_plan_bytes(const td_dock *dock, uint32_t n_req);
int td_plan_create(td_dock *dock, const td_get_req *reqs, uint32_t n_req, void *d_plan,
                   size_t plan_bytes, void *stream, td_plan **out);
int td_plan_destroy(td_plan *plan);
int td_get_many(td_dock *dock, td_plan *plan, void *stream);

/* One buffer serves one RL iteration: forget every table, bitmap and counter; payload bytes
 * and capacities stay. */
int td_reset(td_dock *dock, void *stream);

/* Synchronises `stream`, then copies counters and the error word to *host_out. */
int td_status(td_dock *dock, td_stats *host_out, void *stream);

/* Device address and size of an internal table, for inspection by tests and tools.
 *   which: 0 status u32[n] | 1 len i32[n] (index = class) | 2 off i64[n] (index = class)
 *          3 cursor u64[S] (index = class) | 4 claim bits (index = consumer)
 *          5 consumed bits (index = consumer) | 6 arena or scalar store (index = column) */
int td_debug_table(const td_dock *dock, int which, uint32_t index, void **d_ptr, size_t *bytes);

/* Self-check of the dock's bookkeeping, for tests and for tracking down a misbehaving caller:
 * synchronises `stream`, copies the tables to the host and tests what must hold between any two
 * calls: a stored column implies a reserved row; the rows of a warehouse (the split of the buffer
 * along the batch, "Distributed Transfer Dock Strategy") start on row boundaries, do not overlap
 * and end below the shard's cursor, which stays within the capacity; status words carry no
 * unknown bits; a sample marked served belongs to a claimed group and had every column its
 * consumer needs; the per-column and per-consumer counters equal what the tables say.
 * (While a get is in flight on another stream the claim of a group may be ahead of its served
 * marks; that is not reported.)  violations = 0 means all hold; first_sample names a sample,
 * shard, column or consumer of the first violation found. */
enum {
    TD_BAD_STORED_WITHOUT_ROW = 1u << 0,
    TD_BAD_ROW_PLACEMENT      = 1u << 1,
    TD_BAD_ROW_OVERLAP        = 1u << 2,
    TD_BAD_STATUS_BITS        = 1u << 3,
    TD_BAD_SERVED_UNCLAIMED   = 1u << 4,
    TD_BAD_SERVED_NOT_READY   = 1u << 5,
    TD_BAD_COUNTERS           = 1u << 6
};
typedef struct {
    uint32_t violations, reserved;
    uint64_t first_sample;
    uint64_t stored[32];             /* per column: samples whose status carries its bit */
    uint64_t served[32];             /* per consumer: samples marked served */
    uint64_t arena_elems_used[3];    /* by length class: elements taken by rows, padding included */
} td_validate_report;
int td_debug_validate(td_dock *dock, void *stream, td_validate_report *report);

/* Test hook for the bounded wait of the readiness scan (workflow step 1): a scan tile waits at
 * most poll_limit polls for the tiles ahead of it (0 restores the default, about 2^20), and the
 * tile that draws number skip_tile withholds its descriptor (UINT32_MAX: none), so that the
 * waits of the tiles behind it run out.  Such a get serves nothing, reports
 * TD_ERR_LOOKBACK_TIMEOUT in its result and in the error word, counts n_lookback_timeouts, and
 * hands every claim it made back.  Only this wait is affected; waits on staged copies keep
 * their own limit.  Applies to gets enqueued after the call; not to be called while other host
 * threads are using the dock. */
int td_debug_lookback(td_dock *dock, uint32_t poll_limit, uint32_t skip_tile);

/* Kernels this dock has launched since td_create. */
uint64_t td_launch_count(const td_dock *dock);

/* Per-launch timing of the two copy kernels, the ones that move Eq. 1's payload terms:
 * which = 0 the put scatter, 1 the get gather.  While enabled, each of their launches is
 * bracketed by a pair of CUDA events on the launching stream (host objects; no device memory).
 * td_kernel_timing(dock, enable) clears what was collected and switches collection on or off;
 * td_kernel_timing_read waits for the recorded launches and returns their count and summed
 * device time in milliseconds. */
int td_kernel_timing(td_dock *dock, int enable);
int td_kernel_timing_read(td_dock *dock, int which, uint64_t *launches, double *total_ms);

/* Host-buffer variants: the same workflow steps for a worker whose tensors live in host memory,
 * with the transfers across the bus part of the call (the paper's workers exchange samples
 * between nodes; here the hop is host <-> device).
 * td_put_host: h_indices / h_cu / h_data are HOST arrays (pinned memory makes the copies
 * asynchronous); they are copied into d_stage (device, 256-byte aligned, at least
 * td_put_host_stage_bytes() bytes, not reused until the put has executed) and put from there.
 * td_get_host: runs td_get into the device buffers of dev_out, then copies exactly the valid
 * part of every buffer to the matching HOST pointer of host_out (NULL = skip; host_out->result
 * and host_out->indices are required; col_capacity_elems bounds the host buffers).  It
 * synchronises the stream twice and returns with host_out filled. */
size_t td_put_host_stage_bytes(const td_dock *dock, uint32_t column, uint32_t k, uint64_t data_elems);
int td_put_host(td_dock *dock, uint32_t column, const int32_t *h_indices, uint32_t k,
                const int32_t *h_cu, const void *h_data, uint64_t data_elems,
                void *d_stage, size_t stage_bytes, void *stream);
int td_get_host(td_dock *dock, uint32_t consumer, uint32_t max_samples, const td_get_out *dev_out,
                const td_get_out *host_out, void *stream);
/* The batched calls with host buffers.
 * td_put_many_host: td_put_many whose items' three pointers (named d_* in td_put_item) are HOST
 * arrays here; they are copied, item after item, into d_stage (device, 256-byte aligned, at
 * least the sum of td_put_host_stage_bytes() over the items, not reused until the put has
 * executed) and put from there with one td_put_many; an index or cu array that several items
 * of the call name (same host pointer, same k) is brought over once.
 * td_get_many_host: td_get_many on `plan`, then the valid part of every request's buffers is
 * copied to the matching HOST pointers of host_outs[r] (one entry per request of the plan, in
 * plan order; result and indices required, NULL elsewhere = skip).  All result blocks are
 * fetched behind one synchronisation, all payload behind a second one: two per call however many
 * requests the plan holds, where td_get_host takes two per request.  d_stage (device, 16-byte
 * aligned, td_get_many_host_stage_bytes(plan) bytes, private to the call) is optional: with it
 * the get writes every request's result block, indices, cu_seqlens and advantages a second time,
 * side by side, and one transfer brings them all to the host (the first such call on a plan
 * allocates a pinned host buffer of that size, freed by td_plan_destroy); NULL: one transfer per
 * array and request. */
int td_put_many_host(td_dock *dock, const td_put_item *h_items, uint32_t n_items, void *d_stage,
                     size_t stage_bytes, void *stream);
size_t td_get_many_host_stage_bytes(const td_plan *plan);
int td_get_many_host(td_dock *dock, td_plan *plan, const td_get_out *host_outs, uint32_t n_req, void *d_stage,
                     size_t stage_bytes, void *stream);

/* The communication-volume model of "Distributed Transfer Dock Strategy", in bytes, for sizing a
 * dock or a link (host arithmetic only; no device is touched):
 *   cv        Eq. 1: what one actor-update request takes out of a centralized replay buffer,
 *             G*N*B*(PL + n*SL + M);
 *   tcv       Eq. 2: the total over the last three steps of the replay-buffer workflow,
 *             G*N*B*(2*PL + 3*n*SL + 8*M)                         (Table 1 prints it in GB = 2^30 B);
 *   tcv_dock  Eq. 4: the share of one of S warehouses when C controllers hold the metadata,
 *             G*N*B*(2*PL + 3*n*SL + 8*(C+1)*M) / S               (a double: S need not divide).
 * G prompts, N responses per prompt, PL / SL maximum prompt / response length, n response-length
 * items and M scalars per sample, B bytes per element.  Any out pointer may be NULL.
 * TD_EINVAL: NULL model, S = 0, or a product that does not fit 64 bits. */
typedef struct {
    uint64_t G, N, PL, n, SL, M, B;
    uint64_t C, S;                     /* Eq. 4 only */
} td_model;
int td_model_bytes(const td_model *m, uint64_t *cv, uint64_t *tcv, double *tcv_dock);

/* ---- Operators a model runs on a served batch -------------------------------------------------
 * A get hands a worker state token ids, per-token columns and cu_seqlens; the inference states owe
 * the dock log-probabilities and entropies computed from logits, and the actor update turns the
 * batch into a loss and its gradient (Fig. 2).  These calls are the steps between the batch and the
 * model: the embedding rows of its token ids, the log-probability and entropy of its tokens
 * under the model's logits, the clipped policy loss, and the gradients of all three.
 *
 * They follow the conventions at the top of this file: caller-owned device memory, work enqueued
 * on `stream` only, no synchronisation, no allocation, nothing kept between calls but what a
 * workspace comment says.  The argument structs are host memory, read during the call; `device`
 * is the CUDA device that the pointers belong to (the caller's current device is restored).
 * Sizes that a get decides on the device are read there: where a call takes a td_batch, the number
 * of samples comes from the get's result block, so the host need not know it and the call can
 * stand in a CUDA graph behind the get.  A token id outside [0, vocab) never causes an access
 * outside the operands: a negative id marks a position without a token; an id >= vocab is treated
 * the same and TD_ERR_OOB_INDEX is OR-ed into *status (device, may be NULL; never cleared here).
 * Every sum is in 32 bits or more and in a fixed order: the same call on the same data gives the
 * same bits. */
enum { TD_F16 = 3 };                       /* operands of the operators; a column cannot have it */

/* The row structure of a served batch. */
typedef struct {
    uint32_t max_samples, reserved;
    const int32_t *cu_prompt, *cu_response;   /* device [max_samples + 1], as a get writes them */
    const td_result *result;                  /* device: result->n_samples samples (at most
                                                 max_samples); NULL: exactly max_samples */
} td_batch;

enum { TD_ROWS_TOKEN = 0, TD_ROWS_STREAM = 1 };                    /* td_logprob_args.rows */

/* Log-probability and entropy of tokens under rows of logits x, at temperature tau:
 *   z_v = (x_v - max x) / tau,  S = sum_v e^(z_v),  logprob = z_y - ln S,
 *   entropy = ln S - (sum_v e^(z_v) z_v) / S        (a term with e^(z_v) = 0 is 0).
 * rows = TD_ROWS_TOKEN: logits row t belongs to targets[t]; tokens t < n_tokens, and with a batch
 *   t < cu_response[n_samples].
 * rows = TD_ROWS_STREAM: logits are laid out as the fused token stream (td_get_out.seq), targets
 *   as the packed response column; response token j of sample i is predicted by stream row
 *   cu_prompt[i + 1] + cu_response[i] + j - 1, the position before it (the first token of a
 *   sample without a prompt has none).  Needs batch with both cu arrays.
 * Outputs are in token order, i.e. packed as td_put_back takes them.  A token without a target or
 * without a row gets 0 everywhere.  A row whose logits are all -inf has no distribution: logprob
 * -inf, entropy 0, norm {-inf, 0}.  NaN or +inf in a row makes its outputs NaN.  Outputs of
 * tokens past the batch's end are not written. */
typedef struct {
    const void *logits;                    /* device [n_rows][logits_stride] of dtype */
    int64_t  logits_stride;                /* elements from row to row, >= 0; rows need no alignment */
    int32_t  dtype;                        /* TD_F32 | TD_BF16 | TD_F16 */
    uint32_t vocab, n_rows, n_tokens;      /* n_rows, n_tokens < 2^31; TD_ROWS_TOKEN: n_tokens <= n_rows */
    int32_t  rows;
    float    temperature;                  /* > 0, finite */
    int32_t  device;
    const int32_t *targets;                /* device [n_tokens] */
    const td_batch *batch;                 /* host struct, or NULL (TD_ROWS_TOKEN only) */
    float *logprob;                        /* device [n_tokens]                      required */
    float *norm;                           /* device [n_tokens][2]: {max x, ln S}, for the gradient; or NULL */
    float *entropy;                        /* device [n_tokens], or NULL */
    void  *entropy_bf16;                   /* the same rounded to a TD_BF16 column, or NULL */
    uint32_t *status;
} td_logprob_args;
int td_token_logprob(const td_logprob_args *args, void *stream);

/* Gradient of the above with respect to the logits: with g, h the gradients of a loss with respect
 * to a token's logprob and entropy and p_v = e^(z_v) / S,
 *   grad_v = (g * ([v = y] - p_v) - h * p_v * (ln p_v + entropy)) / tau.
 * Every one of the n_rows rows is written: rows no token belongs to, rows of tokens without
 * a target, and rows whose g and h are both 0 get zeros (their logits are not read); a row whose
 * logits were all -inf gets zeros.  grad_logits may be the logits buffer itself (same pointer, same
 * stride). */
typedef struct {
    const void *logits;
    int64_t  logits_stride;
    int32_t  dtype;
    uint32_t vocab, n_rows, n_tokens;
    int32_t  rows;
    float    temperature;
    int32_t  device;
    const int32_t *targets;
    const td_batch *batch;
    const float *norm;                     /* device [n_tokens][2], from td_token_logprob  required */
    const float *entropy;                  /* device [n_tokens]; required with grad_entropy */
    const float *grad_logprob;             /* device [n_tokens], or NULL (zeros)            */
    const float *grad_entropy;             /* device [n_tokens], or NULL (zeros); one of the two is required */
    void    *grad_logits;                  /* device [n_rows][grad_stride] of dtype  required */
    int64_t  grad_stride;                  /* >= vocab */
    uint32_t *status;
} td_logprob_grad_args;
int td_token_logprob_grad(const td_logprob_grad_args *args, void *stream);

/* Clipped policy loss with a KL term, and its gradient, over the response tokens of a batch.
 * Per counted token, with A the advantage and every log ratio limited to [-30, 30] (its gradient is
 * 0 where the limit acts):
 *   ratio = e^(logprob - old_logprob)                      (old_logprob == NULL: 1, with gradient)
 *   pg    = max(-A ratio, -A clip(ratio, 1 - clip_low, 1 + clip_high));
 *           dual_clip > 0 and A < 0: at most -A dual_clip
 *   d     = ref_logprob - logprob
 *   kl    = -d | d^2 / 2 | e^d - 1 - d                     (TD_KL_K1 | K2 | K3)
 *   loss  = sum over counted tokens of weight * (pg + kl_coef kl - entropy_coef entropy)
 * A token is counted if it lies in a sample's response and its mask byte is not 0; what the
 * other positions of the inputs hold is never used.  weight:
 *   TD_MEAN_TOKENS   1 / norm,               norm = 0: the number of counted tokens
 *   TD_MEAN_SAMPLES  1 / (norm * counted tokens of the sample),  norm = 0: the number of samples
 * (norm > 0 lets micro-batches of one update share a denominator, or divides by a fixed length.)
 * Layout of the per-token arrays: row_width = 0: packed, sample i at cu_response[i]; else padded,
 * sample i at i * row_width (a longer response is cut there), max_samples rows.  Gradients are
 * written at every one of n_tokens positions, 0 where no counted token is, and carry grad_scale.
 * With no counted token at all the loss is 0. */
enum { TD_KL_K1 = 1, TD_KL_K2 = 2, TD_KL_K3 = 3 };
enum { TD_MEAN_TOKENS = 0, TD_MEAN_SAMPLES = 1 };
enum {                                     /* td_policy_args.stats */
    TD_POLICY_LOSS = 0,                    /* the loss                                               */
    TD_POLICY_PG = 1, TD_POLICY_KL = 2, TD_POLICY_ENTROPY = 3,  /* weighted sums of pg, kl, entropy  */
    TD_POLICY_CLIPPED = 4,                 /* share of counted tokens whose pg is held by a clip      */
    TD_POLICY_OLD_KL = 5,                  /* mean of old_logprob - logprob over counted tokens       */
    TD_POLICY_RATIO = 6,                   /* mean ratio over counted tokens                         */
    TD_POLICY_TOKENS = 7,                  /* counted tokens                                         */
    TD_POLICY_STATS = 8
};
typedef struct {
    const td_batch *batch;                 /* cu_response required, cu_prompt unused */
    uint64_t n_tokens;                     /* positions of the per-token arrays; packed: < 2^31, tokens past it are
                                              not counted; padded: max_samples * row_width, < 2^40 */
    uint64_t row_width;
    int32_t  column_dtype;                 /* of old_logprob and ref_logprob: TD_F32 | TD_BF16 */
    int32_t  kl_kind, reduction, device;
    float    clip_low, clip_high;          /* >= 0, clip_low <= 1 */
    float    dual_clip;                    /* 0: off, else > 1 */
    float    kl_coef, entropy_coef, norm, grad_scale;
    uint32_t reserved;
    const float *logprob;                  /* device [n_tokens] */
    const void  *old_logprob;              /* or NULL */
    const void  *ref_logprob;              /* or NULL: no kl term */
    const float *entropy;                  /* or NULL: no entropy term */
    const uint8_t *mask;                   /* or NULL: every response token counts */
    const float *advantages;               /* device [max_samples] */
    float *grad_logprob;                   /* device [n_tokens]            required */
    float *grad_entropy;                   /* device [n_tokens], or NULL (then entropy's term has no gradient) */
    float *stats;                          /* device [TD_POLICY_STATS]     required */
    void  *workspace;                      /* device, 256-byte aligned, zero-filled once after allocation, private
                                              to this call while it is in flight */
    uint64_t workspace_bytes;              /* >= td_policy_loss_workspace_bytes(max_samples) */
} td_policy_args;
size_t td_policy_loss_workspace_bytes(uint32_t max_samples);
int td_policy_loss(const td_policy_args *args, void *stream);

enum { TD_TOKENS_PROMPT = 1, TD_TOKENS_RESPONSE = 2, TD_TOKENS_SEQ = 3 };   /* which tokens of a batch `ids` holds */

/* Embedding rows: out[t] = scale * table[ids[t]], computed in float and rounded once; zeros for a
 * position without a token and, with a batch, for the positions past its tokens (prompt ids,
 * response ids, or the fused stream: `tokens`). */
typedef struct {
    const int32_t *ids;                    /* device [n_tokens] */
    uint32_t n_tokens, vocab, dim;         /* n_tokens < 2^31 */
    int32_t  dtype;                        /* of table and out: TD_F32 | TD_BF16 | TD_F16 */
    const void *table;                     /* device [vocab][table_stride] */
    int64_t  table_stride;                 /* elements; strides >= dim */
    void    *out;                          /* device [n_tokens][out_stride] */
    int64_t  out_stride;
    float    scale;
    int32_t  tokens, device;
    uint32_t reserved;
    const td_batch *batch;                 /* or NULL: all n_tokens */
    uint32_t *status;
} td_embed_args;
int td_embed(const td_embed_args *args, void *stream);

/* Gradient of the above with respect to the table: row v gets scale * (sum of grad_out[t] over
 * the positions with ids[t] = v), summed in float in ascending order of position by blocks of the
 * sorted positions, so that the result does not depend on timing.
 *   accumulate = 0: every row of grad_table is written, 0 where no token is;
 *   accumulate = 1: the sum is added to the rows that occur (in float, rounded once), others keep
 *                   their contents and are not touched.  Float rows are added to where they lie, by
 *                   additions in memory, which take numbers below 2^-126 as zero. */
typedef struct {
    const int32_t *ids;
    uint32_t n_tokens, vocab, dim;
    int32_t  dtype;                        /* of grad_out */
    const void *grad_out;                  /* device [n_tokens][out_stride] */
    int64_t  out_stride;
    int32_t  grad_dtype;                   /* of grad_table: TD_F32 or dtype */
    int32_t  accumulate;
    void    *grad_table;                   /* device [vocab][table_stride] */
    int64_t  table_stride;
    float    scale;
    int32_t  tokens, device;
    uint32_t reserved;
    const td_batch *batch;
    void    *workspace;                    /* device, 256-byte aligned, any contents, private to this call while in flight */
    uint64_t workspace_bytes;              /* >= td_embed_grad_workspace_bytes(n_tokens, vocab, dim) */
    uint32_t *status;
} td_embed_grad_args;
/* Never falls as an argument grows: a workspace for the largest call serves every call with no more
 * positions, vocabulary and columns.  0 where an argument is 2^31 or more. */
size_t td_embed_grad_workspace_bytes(uint32_t n_tokens, uint32_t vocab, uint32_t dim);
int td_embed_grad(const td_embed_grad_args *args, void *stream);

/* ---- A paged key-value cache for generation ----------------------------------------------------
 * What a generation state keeps between two tokens, and the steps on it: keys and values of every
 * token lie in pages of page_size tokens; a table row per sequence names its pages in order, so
 * token j of sequence s lies in page table[s][j / page_size] at place j % page_size; holders[p] counts the
 * table rows that name page p, and a page without a holder is free.  The responses of a GRPO group
 * share their prompt's full pages (td_cache_fork).
 *
 * The conventions of the operators above hold: caller-owned device memory, work on `stream` only, no
 * synchronisation, no allocation.  All of it is device state that the calls read and write in stream order,
 * so that a whole generation step can stand in a CUDA graph; calls on one cache are ordered by the
 * caller (attention calls may overlap each other).  Empty cache: lengths and holders zero; the
 * table may hold anything.  Which sequences a call is about is said by one entry per sequence, so
 * that none is named twice.  A table entry outside [0, n_pages) never causes an access outside the cache: the
 * token or page is passed over and TD_ERR_OOB_INDEX is OR-ed into *status (device, may be NULL,
 * never cleared here).  A sequence whose length lies outside [0, max_pages * page_size] is passed over by a call that
 * has something to do to it, with TD_ERR_BAD_LENGTH. */
typedef struct {
    int32_t  dtype;                        /* TD_F32 | TD_BF16 | TD_F16 */
    uint32_t n_pages, page_size;           /* page_size < 2^16; n_pages * page_size < 2^40 */
    uint32_t n_layers, n_heads, dim;       /* of keys and values, >= 1; n_layers, n_heads < 2^16, dim < 2^16 */
    int64_t  layer_stride, page_stride, token_stride, head_stride;   /* elements, >= 0, the same for both; dim is contiguous.
                                              td_cache_attention takes fewer dims and strides */
    void *keys, *values;                   /* device, layer 0; both NULL: tables only (extend, free) */
    uint32_t max_seqs, max_pages;          /* table rows < 2^24, and entries of a row; max_pages * page_size < 2^31 */
    int32_t *table;                        /* device [max_seqs][max_pages] */
    int32_t *length;                       /* device [max_seqs], tokens */
    int32_t *holders;                      /* device [n_pages] */
    uint32_t *status;
    void    *workspace;                    /* device, 256-byte aligned, any contents, for extend, fork and compact;
                                              private to the call while in flight */
    uint64_t workspace_bytes;              /* >= td_cache_workspace_bytes(n_pages, max_seqs) */
    int32_t  device;
    uint32_t reserved;
} td_cache;
/* Never falls as an argument grows. 0 where an argument is out of range. */
size_t td_cache_workspace_bytes(uint32_t n_pages, uint32_t max_seqs);

/* Room for new tokens: length[s] += add[s], and the pages that takes, the lowest free ones first, in
 * order of s.  add: device [max_seqs], or NULL: one token for every sequence that has any.  cu: device
 * [max_seqs + 1] or NULL: written with the running sum of the tokens given, as td_cache_write takes it.
 * Negative entries and sequences that would pass max_pages get nothing (TD_ERR_BAD_LENGTH).  Where
 * the free pages do not suffice for the whole call nothing is changed, cu is zeros, and
 * TD_ERR_ARENA_FULL is raised; the same with TD_ERR_BAD_LENGTH where cu is given and the call's tokens are
 * 2^31 or more in all.  The last page of a sequence must be its own unless it is full (a fork leaves it so). */
int td_cache_extend(const td_cache *cache, const int32_t *add, int32_t *cu, void *stream);

/* Sequence s becomes a copy of sequence parent[s] (device [max_seqs], negative: none): it holds the parent's
 * full pages too, and a partly filled last page is copied, in every layer, to a page of its own (the
 * lowest free ones, in order of s).  s must be empty, else it is passed over with TD_ERR_DUP_PUT; a
 * parent >= max_seqs is passed over with TD_ERR_OOB_INDEX; a parent that is itself forked to by this
 * call counts as it was before it.  Too few free pages: nothing is changed, TD_ERR_ARENA_FULL. */
int td_cache_fork(const td_cache *cache, const int32_t *parent, void *stream);

/* Sequences with release[s] != 0 (device bytes [max_seqs]; NULL: all) give their pages back and
 * have length 0.  A page that is given back more often than it is held stays free (TD_ERR_DUP_PUT). */
int td_cache_free(const td_cache *cache, const uint8_t *release, void *stream);

/* The U pages that are held move to numbers 0 .. U - 1: the i-th held page with a number >= U, from below,
 * goes to the i-th free number < U, with its contents in every layer and its holders; the tables follow.
 * used: device word, written with U, or NULL.  moved: device [n_pages], written with every page's new number,
 * -1 for a free one, or NULL.  Pages that are left keep their contents. */
int td_cache_compact(const td_cache *cache, uint32_t *used, int32_t *moved, void *stream);

/* Keys and values of new tokens into their pages.  Row t of keys / values belongs to the sequence s with
 * cu[s] <= t < cu[s + 1] (cu: device [max_seqs + 1], from td_cache_extend) and is its token
 * length[s] - (cu[s + 1] - t): the newest tokens, whose room the extend has made.  Rows from n_rows or
 * cu[max_seqs] on are not stored; a row that would be a token before the first is passed over with
 * TD_ERR_BAD_LENGTH. */
typedef struct {
    const td_cache *cache;
    uint32_t layer, n_rows;                /* n_rows < 2^31 */
    const void *keys, *values;             /* device [n_rows][cache->n_heads][cache->dim] of the cache's dtype */
    int64_t  row_stride, head_stride;      /* elements, >= 0; dim is contiguous */
    const int32_t *cu;
} td_cache_write_args;
int td_cache_write(const td_cache_write_args *args, void *stream);

/* Attention of one new token per row over the cache: with kv = h / (n_heads / cache->n_heads),
 *   x_j = scale * q[r][h] . K[j][kv],  lse = ln sum_j e^(x_j),  out[r][h] = sum_j e^(x_j - lse) V[j][kv]
 * over the tokens j of sequence seqs[r] (seqs == NULL: r), with window > 0 its last `window` ones only.
 * Scores, in units of ln 2, their maximum and both sums are float; the weights e^(x_j - reference) are rounded to the cache's
 * type for the product with V (bfloat16, half), where the largest weight of the tokens taken together lies in [1, 2^8]
 * (bfloat16) or [2^7, 2^15] (half): half loses weights below 2^-32 of it, and the sums of 2^8 |V| have to stay within
 * float's range, which bfloat16 values above 10^36 over the number of tokens may pass.
 * A row without a token (seqs[r] < 0, length 0, or every score -inf) has out 0 and lse -inf; seqs[r] >= max_seqs is the
 * same with TD_ERR_OOB_INDEX.  Otherwise the value of a token with a score of -inf is multiplied by 0, so that one
 * that is not finite gives NaN in its column; NaN or +inf among a row's scores makes that row's head NaN.  What lies in a
 * page behind a sequence's last token is never used.
 * Narrower than the other calls on a cache: dim is a multiple of 8 and 256 at most, and keys, values, q and out, and
 * every stride of theirs, are multiples of 16 bytes, else TD_EINVAL.  A cache that is to be attended over is made so.  Float
 * caches: n_rows * cache->n_heads * ceil(n_heads / cache->n_heads / 8) < 2^31.
 * group > 1: rows i * group .. i * group + group - 1 are likely to share leading pages, as the
 * responses of a GRPO group do; the full pages that all of a group's rows (with a token) begin with are then read once
 * for all, in bfloat16 and half, where they hold 64 tokens and spare 2000 reads (tokens times rows less one), no row's
 * window has left the first token, and for every 512 rows (or a like part) of a larger group.  Only time, and the order
 * of sums and so the last bits, depend on it.  Some hundred groups of 8 rows with 600 common tokens, or of 4 with 2000, are
 * faster with it; groups of two rows, and a few groups of 4, are faster with group = 1.
 * Should the products that a group's common tokens are taken with not come in time, the wait for them ends all the same:
 * TD_ERR_COPY_TIMEOUT is raised, out and lse of the heads that needed them are NaN, everything else is right, and the
 * workspace may be used again as it is. */
typedef struct {
    const td_cache *cache;
    uint32_t layer, n_rows, n_heads;       /* n_heads: a multiple of cache->n_heads; n_rows < 2^24 */
    uint32_t group;                        /* >= 1 */
    uint32_t window, reserved;
    float    scale;                        /* scale * log2(e) is finite */
    uint32_t reserved2;
    const int32_t *seqs;                   /* device [n_rows] */
    const void *q;                         /* device [n_rows][n_heads][dim] of the cache's dtype, 16-byte aligned */
    int64_t  q_row_stride, q_head_stride;  /* elements, >= 0, multiples of 16 bytes */
    void    *out;                          /* device, the same shape, type and alignment; rows and heads must not overlap */
    int64_t  out_row_stride, out_head_stride;
    float   *lse;                          /* device [n_rows][n_heads], or NULL */
    void    *workspace;                    /* device, 256-byte aligned, zero-filled once after allocation, private
                                              to this call while it is in flight */
    uint64_t workspace_bytes;              /* >= td_cache_attention_workspace_bytes(n_rows, n_heads, dim) */
} td_cache_attention_args;
/* Never falls as an argument grows. 0 where an argument is out of range.  Room for every form of the call: some 36 MB at
 * dim 128, and (dim + 2) floats per row and head. */
size_t td_cache_attention_workspace_bytes(uint32_t n_rows, uint32_t n_heads, uint32_t dim);
int td_cache_attention(const td_cache_attention_args *args, void *stream);

/* Test hook for that wait: in calls enqueued after it, block number `block` of the kernel takes the wait for its tile-th tile
 * (of 128 common tokens) as run out.  UINT32_MAX: none.  For the whole process. */
int td_debug_cache_wait(uint32_t block, uint32_t tile);

const char *td_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* TD_H */
