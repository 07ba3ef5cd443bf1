/*
 * ef_attention.h - C ABI of the MI355X (gfx950) fused attention library.
 *
 * The library computes the fused attention program of EquiForge (arXiv
 * 2609.12330): for every batch b and query head hq, with kv head
 * hk = hq / (Hq / Hkv) (replication by index, section 3.1 "Replicate"),
 *
 *     s_ij = scale * <q_i, k_j>,   O_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i),
 *     m_i  = max_j s_ij,
 *
 * which is form M0 of figure "attention-rewrites" (section 3). The kernels
 * evaluate it as form M2 of the same figure: the key axis is cut into tiles
 * and a rolling (max, sum, value) reducer is carried over them (section 4.2,
 * repair fusion with h(c, s, s') = c * exp(s - s')). The split-KV entry point
 * additionally stores one reduced state per key partition and combines them
 * in a second kernel (section 3.3 "Collection"; section 4.4 storage rule).
 *
 * Conventions shared by every entry point
 *   - Tensors are dense and row-major with the head dimension innermost:
 *       q  [B][Hq ][Sq ][D] bf16      k, v [B][Hkv][Skv][D] bf16
 *       o  [B][Hq ][Sq ][D] fp32
 *     bf16 is the IEEE binary32 upper half (1-8-7). All pointers are DEVICE
 *     pointers, 16-byte aligned; the caller owns every buffer and keeps it
 *     alive until the stream has passed the call. The library allocates
 *     nothing and keeps no state between calls (apart from the static scratch
 *     of ef_attention_splitkv_noalloc); calls are thread-safe.
 *   - D must be 64 or 128. Hq and Hkv must be >= 1 with Hq % Hkv == 0.
 *     B, Sq and Skv may be 0: with B*Hq*Sq == 0 nothing is written, with
 *     Skv == 0 every output row is 0. Per head, S*D must stay below 2^31.
 *   - causal != 0 applies a bottom-right aligned mask: key j is visible to
 *     query i iff j <= i + (Skv - Sq). A query row that sees no key gets 0.
 *   - scale multiplies the fp32-accumulated q.k products; it must be finite
 *     (0 gives every visible key the same weight). The scaled scores are fp32
 *     values: |scale * q.k| beyond the fp32 range is outside the contract.
 *   - Every call validates its arguments on the host, synchronously, before
 *     anything is enqueued. On an error nothing is launched and no buffer is
 *     written. After validation the work is enqueued on `stream` (a
 *     hipStream_t; NULL is the default stream) and the call returns without
 *     waiting; a launch failure reported by HIP returns EF_ERR_HIP.
 *   - Results are deterministic: the same inputs give bitwise equal outputs.
 *   - Local attention (the *_local entry points; the sliding-window GQA and
 *     attention-sink layers of section 7.3) is causal attention restricted
 *     to a window of `window` keys plus `sinks` sink keys: with
 *     n_i = i + (Skv - Sq), key j is visible to query i iff j <= n_i and
 *     (j > n_i - window or j < sinks). window >= 1, sinks >= 0; a window of
 *     Skv keys or more is plain causal attention. Keys that no query row of
 *     a workgroup can see are not read: the kernels visit the sink keys and
 *     the window and skip the masked middle.
 */
#ifndef EF_ATTENTION_H
#define EF_ATTENTION_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

#define EF_ABI_VERSION 2

typedef enum {
  EF_OK = 0,
  EF_ERR_NULL_POINTER = 1,         /* a required pointer is NULL */
  EF_ERR_INVALID_SHAPE = 2,        /* a negative size, Hq or Hkv < 1, or a head too large */
  EF_ERR_GQA_RATIO = 3,            /* Hq is not a multiple of Hkv */
  EF_ERR_UNSUPPORTED_HEAD_DIM = 4, /* D is not 64 or 128 */
  EF_ERR_MISALIGNED = 5,           /* a pointer is not 16-byte aligned */
  EF_ERR_INVALID_PARTITION = 6,    /* partition_size is not 0 or a positive multiple of 64, or
                                      it gives more than 65535 partitions */
  EF_ERR_WORKSPACE_TOO_SMALL = 7,  /* workspace is NULL or smaller than required */
  EF_ERR_INVALID_SCALE = 8,        /* scale is NaN or infinite */
  EF_ERR_HIP = 9,                  /* HIP reported an error when the work was enqueued */
  EF_ERR_INVALID_MASK = 10,        /* local attention: window < 1 or sinks < 0 */
  EF_ERR_INVALID_DIFF = 11,        /* differential attention: lambda_init or eps not finite, or eps < 0 */
  EF_ERR_INVALID_SPLIT = 12,       /* d_splits not 1, 2 or 4, or more than 8 query rows per kv head */
  EF_ERR_SCRATCH_TOO_SMALL = 13,   /* the problem needs more than EF_STATIC_SCRATCH_BYTES of scratch */
  EF_ERR_INVALID_BLOCKS = 14,      /* block_size not 64 or 128, more than EF_MAX_BLOCKS blocks, or topk,
                                      sink_blocks, local_blocks or new_keys out of range */
  EF_ERR_INVALID_PAGES = 15,       /* page not 16, 32, 64, 128 or 256, fewer than one page, a table width
                                      out of range, or an unknown cache format */
  EF_ERR_INVALID_ROPE = 16         /* rot not a multiple of 16 in 16 .. D, or an amplitude not finite */
} ef_status;

/* Version of this ABI (EF_ABI_VERSION). */
int ef_abi_version(void);

/* Static, NUL-terminated description of a status code; never NULL. */
const char* ef_status_string(int status);

/*
 * Single-pass attention: form M2 of figure "attention-rewrites". The query
 * rows that share a kv head are tiled along the query axis (grid axis m), each
 * workgroup carries the rolling reducer over all key tiles it can see and
 * writes O = value / sum once at the end (section 6.1: output-tile axes map
 * to the grid, reduction axes to an in-workgroup loop).
 *   q, k, v, o : device buffers in the layouts above.
 *   B, Hq, Hkv, Sq, Skv, D, scale, causal : as above.
 *   stream     : hipStream_t or NULL.
 */
ef_status ef_attention_fwd(const void* q, const void* k, const void* v, float* o,
                           int B, int Hq, int Hkv, int Sq, int Skv, int D,
                           float scale, int causal, void* stream);

/*
 * ef_attention_fwd with local attention (causal mask, sliding window of
 * `window` keys, `sinks` sink keys; see the conventions above). Each
 * workgroup reads the key tiles of the sink run and of its rows' windows
 * only; both runs feed one rolling reducer, so sink and window keys share one
 * softmax normalisation (section 7.3, attention sinks).
 * Returns EF_ERR_INVALID_MASK when window < 1 or sinks < 0.
 */
ef_status ef_attention_fwd_local(const void* q, const void* k, const void* v, float* o,
                                 int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                 float scale, int window, int sinks, void* stream);

/*
 * Partition size, in keys, that ef_attention_splitkv uses for these sizes:
 * `partition_size` itself when it is positive, else the library's choice
 * (the candidate ef_attention_splitkv_modeled_us rates fastest).
 * Returns 0 when the arguments are invalid.
 */
int ef_attention_splitkv_partition_size(int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                        int partition_size);

/*
 * Bytes of workspace ef_attention_splitkv needs for these sizes (0 when the
 * arguments are invalid or nothing is computed). With rows = B*Hq*Sq,
 * P = ceil(Skv / T) and T the resolved partition size, the workspace holds
 *     counters [512][64] uint32 at byte 0 (EF_COUNTER_REGION_BYTES)
 *     m   [rows][P]    fp32 at byte  C = EF_COUNTER_REGION_BYTES
 *     l   [rows][P]    fp32 at byte  C + A, A = round_up(rows*P*4, 256)
 *     acc [rows][P][D] fp32 at byte  C + 2*A
 * with row = (b*Hq + hq)*Sq + sq: a reference point m for the scaled scores
 * s of the row's visible keys in partition p (natural-log units; at most the
 * partition maximum and within 8*ln(2) of it), l = sum exp(s - m) and
 * acc = sum exp(s - m) * v. (m, l, acc) and (m', l*e^(m-m'), acc*e^(m-m'))
 * describe the same state. A partition with no visible key holds the reducer
 * identity (-inf, 0, 0). The counters are arrival counters of the fused
 * combine (see ef_attention_splitkv): word 0 of each 256-byte slot
 * counters[b*Hkv + hk] serves one (batch, kv head); the rest is padding. The
 * counter region has the same place and size for every problem, and no
 * partial state is ever stored in it.
 */
#define EF_COUNTER_REGION_BYTES ((size_t)512 * 256)

size_t ef_attention_splitkv_workspace_size(int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                           int partition_size);

/*
 * Split-KV attention for decode-shaped problems (few query rows per kv head,
 * long key axis). The key axis is cut into P partitions of T keys; one
 * workgroup per (partition, kv head, batch) reads its K/V slice once, serves
 * all Hq/Hkv * Sq query rows of that kv head, and stores the reduced state
 * (m, l, acc) of every row in the workspace (the Collection of section 3.3
 * and the storage rule of section 4.4). A second kernel combines the P states
 * of each row with the same reducer and writes o (section 4.1, reduction
 * refinement along K; section 4.2, repair fusion).
 *   partition_size   : T in keys; 0 lets the library choose; otherwise a
 *                      positive multiple of 64.
 *   workspace        : device buffer of at least
 *                      ef_attention_splitkv_workspace_size(...) bytes,
 *                      16-byte aligned; on return (stream-ordered) it holds
 *                      the partial states in the layout documented there.
 *                      Its counter region (the first EF_COUNTER_REGION_BYTES)
 *                      must be zero before the first call that uses it
 *                      (zero-fill the new buffer once); every completed call
 *                      leaves it zero again, so a workspace serves any number
 *                      of calls of any shapes whose workspace fits in it, in
 *                      stream order. Calls that overlap in time must not share
 *                      a workspace.
 *   workspace_bytes  : its size in bytes.
 * When G*Sq <= 4, P <= 64 and B*Hkv <= 512 the combine runs inside the
 * producer: the last workgroup of each (batch, kv head) to store its state,
 * found with the group's arrival counter, combines that group's rows and
 * resets the counter (one kernel instead of two). Otherwise a separate combine
 * kernel follows. A counter that is not zero when the call begins (a counter
 * region never cleared, or written over) cannot tell which workgroup is last:
 * from P on, the producer fills that group's output rows with NaN rather than
 * combine states that may be stale; a value of 1 .. P - 1 looks like arrivals
 * of the call itself and leaves the rows undefined, in this call and in later
 * ones. Clearing the region makes the workspace good again.
 * Other arguments as for ef_attention_fwd.
 */
ef_status ef_attention_splitkv(const void* q, const void* k, const void* v, float* o,
                               int B, int Hq, int Hkv, int Sq, int Skv, int D,
                               float scale, int causal, int partition_size,
                               void* workspace, size_t workspace_bytes, void* stream);

/*
 * Split-KV attention with local attention (causal mask, window, sinks; see
 * the conventions above). The keys any query row of a (batch, kv head) can
 * see lie in two runs: the sink run [0, La), La = min(round_up(sinks, 64),
 * Skv), and the window run [Bs, Skv), Bs = max(La, round_down(max(0,
 * Skv - Sq - window + 1), 64)). The partitions of T keys cut the
 * concatenation of the two runs, Lv = La + Skv - Bs keys, so P = ceil(Lv / T)
 * and no workgroup is spent on the masked middle. Workspace layout, counters
 * and the fused-combine rule are those of ef_attention_splitkv with this P
 * (partition p covers concatenated keys [p*T, p*T + T)).
 * Returns EF_ERR_INVALID_MASK when window < 1 or sinks < 0.
 */
ef_status ef_attention_splitkv_local(const void* q, const void* k, const void* v, float* o,
                                     int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                     float scale, int window, int sinks, int partition_size,
                                     void* workspace, size_t workspace_bytes, void* stream);

/*
 * Partition size and workspace bytes of ef_attention_splitkv_local, as for
 * the causal entry points but over the Lv keys of the two visible runs.
 * Return 0 when the arguments are invalid (including window < 1 or sinks < 0).
 */
int ef_attention_splitkv_local_partition_size(int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                              int window, int sinks, int partition_size);
size_t ef_attention_splitkv_local_workspace_size(int B, int Hq, int Hkv, int Sq, int Skv,
                                                 int D, int window, int sinks,
                                                 int partition_size);

/*
 * The producer step of ef_attention_splitkv alone: the same validation and
 * the same kernels, writing only the partial states into the workspace
 * (layout of ef_attention_splitkv_workspace_size). Combining them with
 * ef_attention_combine gives ef_attention_splitkv's output; partial states of
 * disjoint key ranges (e.g. computed on different devices, each over its own
 * slice of the key axis) may be concatenated along P before the combine,
 * since the combine applies the same reducer to any set of stored states.
 */
ef_status ef_attention_splitkv_partials(const void* q, const void* k, const void* v,
                                        int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                        float scale, int causal, int partition_size,
                                        void* workspace, size_t workspace_bytes, void* stream);

/*
 * The combine step alone, over caller-provided fp32 partial states:
 *   m [rows][P], l [rows][P], acc [rows][P][D] (device, 16-byte aligned),
 *   o [rows][D] fp32 output.
 * For each row: M = max_p m_p, w_p = exp(m_p - M) (0 where m_p = -inf),
 * o = (sum_p w_p acc_p) / (sum_p w_p l_p), and o = 0 when M = -inf
 * (section 4.2, the fused reducer applied to stored states).
 * rows >= 0, P >= 1, D in {64, 128}.
 */
ef_status ef_attention_combine(const float* m, const float* l, const float* acc, float* o,
                               int rows, int num_partitions, int D, void* stream);

/*
 * Modelled duration in microseconds of one split-KV call with
 * `partition_size` keys per partition (window = sinks = 0 for the causal or
 * full entry point; a local window otherwise). The model is the roofline rule
 * of section 6.2, static family ranking (over legal schedules, minimise the
 * largest work/throughput ratio over resources): the larger of the HBM time
 * (K/V, q, o and the partial states written and read) and one workgroup's
 * streaming time times the rounds of workgroups the chip holds, plus the
 * combine, with rates measured on MI355X. With partition_size = 0 the
 * split-KV entry points take the candidate (64, 128, 256, 512, ... keys, and
 * one partition holding every key) this model rates fastest.
 * Returns a negative value for invalid arguments. (With 3 or 4 query rows per
 * kv head and at most 512 partitions over all heads the producer runs four waves
 * per partition; the model rates one, which is 1.1 to 3 times slower.)
 */
double ef_attention_splitkv_modeled_us(int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                       int window, int sinks, int partition_size);

/*
 * Query rows per workgroup of the matrix-core kernel for these sizes, as the
 * entry points choose them (64 or 128; the Hq/Hkv query heads of a kv head
 * are packed into its rows). The choice follows the roofline rule of section
 * 6.2 over the legal values: each is charged the larger of its matrix work
 * (rows padded to whole workgroups) over the bf16 peak and its global-memory
 * traffic (the K/V that every row tile stages, plus q and o) over the HBM
 * peak; the smallest wins, and with equal times the one with less matrix
 * work. `keys`: the keys a row tile streams (Skv for a full or causal
 * prefill, the partition size in a split-KV call). Returns 0 for invalid
 * sizes or keys < 0. The split-KV calls run what this returns; a single-pass
 * launch too small to fill the chip runs 64-row tiles whose keys two groups of
 * waves share instead, which ef_attention_fwd_schedule reports.
 */
int ef_attention_rows_per_workgroup(int B, int Hq, int Hkv, int Sq, int Skv, int D, int keys);

/*
 * How ef_attention_fwd (window = 0) or ef_attention_fwd_local runs these sizes:
 * the query rows per workgroup (64 or 128), plus EF_SCHEDULE_KEY_SPLIT when two
 * groups of waves share a workgroup's key tiles, plus EF_SCHEDULE_LONGEST_FIRST
 * when row tiles run longest first over the heads of a die instead of head by
 * head. Returns 0 for invalid sizes and when there is nothing to attend.
 */
#define EF_SCHEDULE_KEY_SPLIT 256
#define EF_SCHEDULE_LONGEST_FIRST 512
int ef_attention_fwd_schedule(int B, int Hq, int Hkv, int Sq, int Skv, int D, int causal,
                              int window, int sinks);

/*
 * Measures the best partition size for these inputs on this device: the six
 * candidates the model rates fastest (among those whose workspace fits in
 * workspace_bytes) are timed by successive halving (section 6.3: every
 * remaining candidate runs, the faster half stays, the repetitions double)
 * and the winner is written to *partition_size. window = 0 selects the
 * full/causal path (causal as given; sinks must be 0), window > 0 the local
 * path. Runs the split-KV call many times on `stream` (o and the workspace
 * are overwritten), waits for it with HIP events, and so cannot be captured
 * in a graph. Errors as for the split-KV entry points; EF_ERR_NULL_POINTER
 * when partition_size is NULL.
 */
ef_status ef_attention_splitkv_tune(const void* q, const void* k, const void* v, float* o,
                                    int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                    float scale, int causal, int window, int sinks,
                                    void* workspace, size_t workspace_bytes, void* stream,
                                    int* partition_size);

/*
 * Differential attention (section 7.3, the differential attention layer of
 * the cited differential transformer): two attention branches over one value
 * tensor,
 *   A1 = attention(q1, k1, v),  A2 = attention(q2, k2, v)
 * (same scale, causal flag and grouped-query mapping as ef_attention_fwd),
 * mixed with the learned weight
 *   lambda = exp(<lambda_q1, lambda_k1>) - exp(<lambda_q2, lambda_k2>) + lambda_init
 * and normalised per head and query row over the head dimension:
 *   y = A1 - lambda * A2
 *   o = (1 - lambda_init) * norm_weight * y / sqrt(mean(y^2) + eps),
 * and o = 0 for a row where mean(y^2) + eps is 0 (y = 0 with eps = 0). The
 * weight, the difference and the normalisation are applied as the branches'
 * outputs are formed, so no A1 tensor is written.
 *   q1, q2 : [B][Hq][Sq][D] bf16; k1, k2, v : [B][Hkv][Skv][D] bf16;
 *   o      : [B][Hq][Sq][D] fp32, also used to hold A2 between the branches of
 *            a split call.
 *   lambda_q1, lambda_k1, lambda_q2, lambda_k2, norm_weight : [D] fp32 device
 *            buffers, shared by all heads; norm_weight 16-byte aligned.
 *   lambda_init, eps : finite, eps >= 0 (else EF_ERR_INVALID_DIFF).
 *   partition_size : 0 (the library's choice: one partition when the key axis
 *            is short or the query rows fill whole rounds of the chip, else as
 *            for ef_attention_splitkv) or a positive multiple of 64. When the resolved partition covers every
 *            key both branches run in one single-pass launch and the workspace
 *            is not used (it may be NULL); otherwise each branch runs the split-KV
 *            producer into `workspace` (ef_diff_attention_workspace_size bytes,
 *            16-byte aligned, reused by both branches) and its combine. With
 *            partition_size 0 and 192 or more tiles of 128 query rows (B * Hkv *
 *            ceil(Sq * Hq/Hkv / 128), Sq * Hq/Hkv > 64) a missing, small or
 *            misaligned workspace means one launch too.
 * Other errors as for ef_attention_splitkv; all buffers are caller-owned and
 * the call is asynchronous on `stream`.
 */
ef_status ef_diff_attention(const void* q1, const void* q2, const void* k1, const void* k2,
                            const void* v, float* o, const float* lambda_q1,
                            const float* lambda_k1, const float* lambda_q2,
                            const float* lambda_k2, const float* norm_weight, float lambda_init,
                            float eps, int B, int Hq, int Hkv, int Sq, int Skv, int D,
                            float scale, int causal, int partition_size, void* workspace,
                            size_t workspace_bytes, void* stream);

/*
 * Workspace bytes ef_diff_attention needs for this shape and partition_size:
 * 0 when the resolved partition covers every key (single pass) with and without
 * a causal mask, else the split-KV workspace of one branch. Returns 0 for invalid arguments too.
 */
size_t ef_diff_attention_workspace_size(int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                        int partition_size);

/*
 * Decode with an output-channel split (section 7.2: at batch 1 the paper's
 * selected decode kernel gives each head two blocks that compute the same
 * scores and softmax and write different halves of the output, with no merge
 * kernel; the N parallel refinement of the p.V product, section 4.1 and table
 * "rules"). Each key
 * partition of each (batch, kv head) is evaluated by d_splits workgroups:
 * every one reads the partition's K rows and recomputes the scores, and reads,
 * accumulates and writes only its D/d_splits value channels. The output is
 * ef_attention_splitkv's.
 *   q, k, v, o, B, Hq, Hkv, Sq, Skv, D, scale, causal : as ef_attention_splitkv;
 *            at most 8 query rows per kv head ((Hq/Hkv)*Sq <= 8), else
 *            EF_ERR_INVALID_SPLIT.
 *   d_splits : 1, 2 or 4 (else EF_ERR_INVALID_SPLIT).
 *   partition_size : as ef_attention_splitkv (0 = the model's choice). When it
 *            covers every key (one partition) each workgroup writes its
 *            channels of o directly: no workspace (it may be NULL) and no
 *            merge. Otherwise the workspace (ef_attention_decode_dsplit_workspace_size
 *            bytes, 16-byte aligned, counters zero on entry and left zero, as for
 *            ef_attention_splitkv; counter slot (b*Hkv + hk)*d_splits + slice)
 *            holds the states, which every channel slice combines for its own
 *            channels (in the producer when P <= 64 and B*Hkv*d_splits <= 512).
 */
ef_status ef_attention_decode_dsplit(const void* q, const void* k, const void* v, float* o,
                                     int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                     float scale, int causal, int d_splits, int partition_size,
                                     void* workspace, size_t workspace_bytes, void* stream);

/*
 * Workspace bytes of ef_attention_decode_dsplit: 0 with one partition, else
 * the split-KV layout (the same counter region and states). 0 for invalid
 * arguments too.
 */
size_t ef_attention_decode_dsplit_workspace_size(int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                                 int d_splits, int partition_size);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc):
 * ef_attention_splitkv with the workspace replaced by a scratch array of
 * static device storage that the library holds, EF_STATIC_SCRATCH_BYTES per
 * device. The array is reserved when the library's code object is loaded on
 * a device and held until the process ends; the call itself allocates
 * nothing. The first call on a device also looks up that device's copy of
 * the array (a host-side query, not a stream operation), so make it outside
 * graph capture.
 *   Arguments, validation and output: as ef_attention_splitkv, without
 *   `workspace` and `workspace_bytes`. Returns EF_ERR_SCRATCH_TOO_SMALL, with
 *   nothing enqueued, when ef_attention_splitkv_workspace_size(...) for these
 *   arguments exceeds EF_STATIC_SCRATCH_BYTES (every other argument error is
 *   reported first), and EF_ERR_HIP when the scratch array cannot be found on
 *   the current device.
 * Every call on one device shares that device's scratch, which keeps the last
 * call's partial states: calls that overlap in time on one device race with
 * each other and must be ordered (e.g. issued on one stream). The arrival
 * counters in the scratch start at zero and every completed call leaves them
 * at zero.
 */
#define EF_STATIC_SCRATCH_BYTES ((size_t)32 << 20)

ef_status ef_attention_splitkv_noalloc(const void* q, const void* k, const void* v, float* o,
                                       int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                       float scale, int causal, int partition_size,
                                       void* stream);

/*
 * Long contexts: block-sparse attention and shared prefixes
 *
 * The entry points below serve long contexts: attention over selected blocks of
 * the key axis (the blocks' summaries, the choice of each query's blocks, the
 * attention over them) and attention of a batch of sequences over one prefix.
 * They follow the conventions at the top of this file, and in addition:
 *   - lengths : device buffer of B int32, or NULL. Sequence b has
 *     len_b = lengths[b] valid keys (clamped to [0, Skv]); Skv, the extent of its
 *     buffers, is then a capacity. With NULL every sequence has Skv keys. What lies
 *     behind a sequence's length is never read. Keys and values below it must be
 *     finite. A query that is not makes those of its own attention rows NaN that see
 *     a key, and no others.
 *   - Query i of sequence b sits at key n_i = i + len_b - Sq of its sequence (its
 *     queries are its last Sq positions); a negative n_i sees nothing.
 *   - o is bf16, the type the next product takes: one rounding of an fp32 result.
 *   - block_size is 64 or 128 keys; block n holds the keys [n * block_size,
 *     (n + 1) * block_size), and a key axis of Skv keys has
 *     NB = ceil(Skv / block_size) <= EF_MAX_BLOCKS blocks.
 */
#define EF_MAX_BLOCKS 16000
#define EF_MAX_TOPK 256

/*
 * Summary of the blocks of a key cache: the mean of each block's valid keys,
 *   summary[b][h][n] = sum over the valid keys j of block n of k[b][h][j] / their number,
 * and 0 for a block without a valid key. The sum is fp32 and rounded to bf16 once.
 *   k        : [B][Hkv][Skv][D] bf16;  summary : [B][Hkv][NB][D] bf16.
 *   new_keys : 0 writes every block. A positive number writes only the blocks that
 *              hold one of each sequence's last new_keys valid keys, and leaves the
 *              others as they are: after a decode step appended a key to every
 *              sequence, new_keys = 1 brings the summaries up to date.
 * Errors: EF_ERR_INVALID_BLOCKS for block_size, NB or new_keys < 0; others as for
 * ef_attention_fwd.
 */
ef_status ef_block_summary(const void* k, const int* lengths, void* summary, int B, int Hkv,
                           int Skv, int D, int block_size, int new_keys, void* stream);

/*
 * Choice of the blocks each query attends to. For query i of sequence b and kv
 * head h, cur = floor(n_i / block_size) is the query's own block.
 *   - n_i < 0: no block.  cur + 1 <= topk: the blocks 0 .. cur.
 *   - Otherwise topk blocks of 0 .. cur: the first sink_blocks, the last
 *     local_blocks (up to cur, which is always one of them), and of the others
 *     those with the largest score
 *       score(n) = max over the Hq/Hkv query heads g of h of <q[b][g][i], summary[b][h][n]>,
 *     ties to the lower index; a NaN product counts as -inf.
 * The choice is that of exact arithmetic: where two scores are too close for fp32
 * to tell apart they are formed again in 64 bits. (Scores beyond the fp32 range
 * are outside the contract.) The result does not depend on scheduling. What a
 * summary at or behind a query's local blocks holds does not matter, a partial last
 * block's least of all.
 *   q       : [B][Hq][Sq][D] bf16;  summary : [B][Hkv][NB][D] bf16, NB of Skv keys.
 *   blocks  : [B][Hkv][Sq][topk] int32: ascending block indices, then -1.
 *   topk    : 1 .. EF_MAX_TOPK, at least sink_blocks + local_blocks.
 *   sink_blocks >= 0, local_blocks >= 1.
 * Errors: EF_ERR_INVALID_BLOCKS for block_size, NB, topk, sink_blocks, local_blocks;
 * EF_ERR_INVALID_SHAPE also for more queries of one sequence than a launch takes (Hkv * Sq of
 * 2^22 and more may be); others as for ef_attention_fwd.
 */
ef_status ef_block_select(const void* q, const void* summary, const int* lengths, int* blocks,
                          int B, int Hq, int Hkv, int Sq, int Skv, int D, int block_size,
                          int topk, int sink_blocks, int local_blocks, void* stream);

/*
 * Attention over selected blocks: query i of sequence b and query head hq sees the
 * keys j <= n_i whose block is in the list of (b, hq / (Hq/Hkv), i). A row without a
 * visible key gets 0.
 *   blocks : [B][Hkv][Sq][topk] int32, 16-byte aligned, as ef_block_select writes it
 *            or any other choice: the order does not matter, an entry outside
 *            0 .. floor(n_i / block_size) is passed over, a repeated one counts once.
 *   topk   : 1 .. EF_MAX_TOPK.
 *   o      : [B][Hq][Sq][D] bf16.
 *   workspace : ef_attention_blocks_workspace_size(...) bytes, 16-byte aligned (may
 *            be NULL where that is 0), with the counter region of
 *            ef_attention_splitkv's workspace at its start: zero before the first
 *            call that uses it, left zero by every completed call. One workspace
 *            serves any number of calls of these and the split-KV entry points, in
 *            stream order; calls that overlap in time must not share one, and neither
 *            must two captured graphs that may run at the same time. A counter that
 *            was not zero is as in ef_attention_splitkv: NaN rows from the number of
 *            the workgroups that share a row (16 at most) on, undefined ones below.
 * Work and traffic grow with the union of the lists of about 64 * Hkv / Hq neighbouring
 * queries, which is little more than one list where neighbours choose alike.
 * Errors: EF_ERR_INVALID_BLOCKS for block_size, NB or topk; others as for
 * ef_attention_splitkv.
 */
ef_status ef_attention_blocks(const void* q, const void* k, const void* v, const int* blocks,
                              const int* lengths, void* o, int B, int Hq, int Hkv, int Sq,
                              int Skv, int D, float scale, int block_size, int topk,
                              void* workspace, size_t workspace_bytes, void* stream);

/* Workspace bytes of ef_attention_blocks; 0 for invalid arguments too. */
size_t ef_attention_blocks_workspace_size(int B, int Hq, int Hkv, int Sq, int Skv, int D,
                                          int block_size, int topk);

/*
 * Attention of a batch over one shared prefix: the keys of sequence b are the Lp keys
 * of the prefix, the same for all sequences, followed by its len_b own ones. With
 * causal != 0 query i sees the keys up to its own place, Lp + n_i, of this
 * concatenation (a place before its first key: none, and the row is 0); otherwise it
 * sees them all. A prefix key is read once for every 128 rows (Hq/Hkv * Sq of each
 * sequence) of all sequences, instead of once per sequence; where a sequence's own rows
 * fill such tiles and the batch's the chip, once for every 128 of a sequence's rows.
 *   k_prefix, v_prefix : [Hkv][Lp][D] bf16;  k, v : [B][Hkv][Skv][D] bf16.
 *   o         : [B][Hq][Sq][D] bf16.
 *   Lp, Skv   : either may be 0.
 *   workspace : as for ef_attention_blocks, ef_attention_shared_prefix_workspace_size(...)
 *               bytes.
 * Errors as for ef_attention_splitkv.
 */
ef_status ef_attention_shared_prefix(const void* q, const void* k_prefix, const void* v_prefix,
                                     const void* k, const void* v, const int* lengths, void* o,
                                     int B, int Hq, int Hkv, int Sq, int Lp, int Skv, int D,
                                     float scale, int causal, void* workspace,
                                     size_t workspace_bytes, void* stream);

/* Workspace bytes of ef_attention_shared_prefix; 0 for invalid arguments too. */
size_t ef_attention_shared_prefix_workspace_size(int B, int Hq, int Hkv, int Sq, int Lp, int Skv,
                                                 int D);

/*
 * Serving: rotary positions, a paged key-value cache, packed sequences
 *
 * What a serving loop does around its matrix products: rotate the queries and keys of new
 * tokens, append keys and values to a cache in pages, attend to the cache (one or a few new
 * tokens of each sequence) or to packed rows (prompts, or chunks of them). Conventions as at
 * the top of this file, but for these:
 *   - Packed rows [T][H][D]: the rows of sequence b are starts[b] .. starts[b + 1] - 1.
 *     starts is a device buffer of B + 1 ascending int32. Rows in front of the first sequence or
 *     behind the last one belong to none: outputs there are left as they were. Starts out of
 *     [0, T] count as clamped to it.
 *   - The new tokens of a sequence are the last ones of its keys: with n_b new tokens and
 *     len_b = lengths[b] keys, new token i stands at position len_b - n_b + i.
 *   - A cache holds k and v, each [pages][Hkv][page][D]: bf16 (EF_CACHE_BF16), or e4m3 codes
 *     (EF_CACHE_E4M3) beside an fp32 scale for each row, [pages][Hkv][page]. Row at of
 *     page table[b][n] is position n * page + at of sequence b; table is a device buffer
 *     [B][width] of int32. Entries behind a sequence's last page are not read. page is 16, 32,
 *     64, 128 or 256.
 *   - An entry outside 0 .. pages - 1 names no page: a token that belongs there is not written,
 *     is read as NaN, and makes the attention rows that see it NaN.
 *   - Caches may have any size (offsets of 64 bits). Keys and values that a row may see must be
 *     finite, and so must the fp32 sums over them; a query that is not makes its own rows NaN
 *     that see a key.
 */
#define EF_CACHE_BF16 0
#define EF_CACHE_E4M3 1

/*
 * Rotary positions: of every row x[t][h] the pairs (a, b) among its first `rot` elements are
 * turned by the angle 2 pi positions[t] turns[i] of pair i and multiplied by amplitude,
 *   y_a = amplitude (x_a cos - x_b sin),  y_b = amplitude (x_b cos + x_a sin);
 * the others are copied. Pair i is (2 i, 2 i + 1) with interleaved != 0, else (i, i + rot / 2).
 * transpose != 0 applies the transposed map (the angle negated), which takes the gradient of y
 * to the gradient of x.
 *   x, out    : [T][H][D] bf16; they may be the same buffer, but not overlap otherwise.
 *   positions : [T] int32, any value.
 *   turns     : [rot / 2] double, device, 16-byte aligned: turns (of 2 pi) per position. Angles
 *               are formed in 64 bits (with turns of at most 1 / 2 pi they are off by 2^-25 turns at
 *               most); amplitude cos and amplitude sin are rounded to fp32, and so is each product
 *               and sum, and the result to bf16.
 *   rot       : a multiple of 16, 16 .. D.
 * Errors: EF_ERR_INVALID_ROPE; others as for ef_attention_fwd.
 */
ef_status ef_rope(const void* x, const int* positions, const double* turns, void* out, int T,
                  int H, int D, int rot, int interleaved, double amplitude, int transpose,
                  void* stream);

/*
 * Appends the new tokens of every sequence to a cache: k[t] rotated and v[t] go to the row of
 * the token's position, and with q the rotated queries to q_out, in one launch.
 *   k, v     : [T][Hkv][D] bf16;  q, q_out : [T][Hq][D] bf16, q_out may be q; or both NULL (Hq
 *              is then 0 or a multiple of Hkv).
 *   turns    : as for ef_rope, or NULL: nothing is rotated (rot, interleaved and amplitude are
 *              ignored).
 *   lengths  : [B] int32, device: the keys of every sequence, its new tokens among them.
 *   starts   : [B + 1] int32, or NULL: every sequence has T / B new tokens (T % B == 0).
 *   k_scale, v_scale : [pages][Hkv][page] fp32 with EF_CACHE_E4M3 (ignored otherwise).
 * A row of 8 bits is held as codes x / s, rounded to e4m3 once; s is the smallest power of two,
 * at least 2^-100, that brings the row's largest finite magnitude to 448 at most. Elements that
 * are not finite become NaN. A token in front of position 0 or behind the table is not written.
 * Two tokens must not have the same row of the cache.
 */
ef_status ef_cache_write(const void* k, const void* v, const void* q, const double* turns,
                         void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                         const int* table, const int* lengths, const int* starts, void* q_out,
                         int T, int B, int Hq, int Hkv, int D, int pages, int page, int width,
                         int format, int rot, int interleaved, double amplitude, void* stream);

/*
 * The cached keys and values of every sequence as packed bf16 rows: position i of sequence b
 * goes to row starts[b] + i, starts[b + 1] - starts[b] of them (at most width * page; further
 * rows are NaN, as those of entries that name no page). bf16 rows are copied; 8-bit ones
 * are code times scale, which is exact for scales that ef_cache_write makes.
 *   k_out, v_out : [T][Hkv][D] bf16.
 */
ef_status ef_cache_read(const void* k_cache, const void* v_cache, const float* k_scale,
                        const float* v_scale, const int* table, const int* starts, void* k_out,
                        void* v_out, int T, int B, int Hkv, int D, int pages, int page, int width,
                        int format, void* stream);

/*
 * Attention of new tokens over a paged cache that holds them: row (t, hq) of new token i of
 * sequence b sees the positions up to its own, len_b - n_b + i. A row that sees none is 0.
 *   q, o      : [T][Hq][D] bf16; o may be q.
 *   lengths   : [B] int32, clamped to [0, width * page].
 *   starts    : [B + 1] int32, or NULL: every sequence has T / B new tokens (T % B == 0).
 *   max_queries : most new tokens of a sequence; of one that has more, only the first
 *               max_queries rows are written. With starts = NULL at least T / B.
 *   workspace : ef_attention_paged_workspace_size(...) bytes, 16-byte aligned, with the
 *               counter region of ef_attention_splitkv's workspace at its start; the same rules.
 *               Its size does not depend on lengths, and one for larger T, B and max_queries
 *               serves smaller ones.
 * Limits beside those of the other calls: B (width page / 64 + 32) < 2^31 (units of work that are
 * counted in 32 bits), and max_queries Hq / 32 <= 2^23 (workgroups of a launch).
 * The keys of all sequences are dealt evenly to the compute units, whatever their lengths. (Not so
 * the rows: 32 of a kv head share a walk, and the more there are, the fewer workgroups a walk has.
 * A chunk of hundreds of tokens and single tokens of other sequences take less time in two calls.)
 * Results depend on how they are dealt, that is on the other sequences of the call, in the last
 * bits; the same call gives the same bits.
 */
ef_status ef_attention_paged(const void* q, const void* k_cache, const void* v_cache,
                             const float* k_scale, const float* v_scale, const int* table,
                             const int* lengths, const int* starts, void* o, int T, int B, int Hq,
                             int Hkv, int D, int max_queries, int pages, int page, int width,
                             int format, float scale, void* workspace, size_t workspace_bytes,
                             void* stream);

/* Workspace bytes of ef_attention_paged; 0 for invalid arguments too. */
size_t ef_attention_paged_workspace_size(int T, int B, int Hq, int Hkv, int D, int max_queries);

/*
 * Attention of packed sequences of any lengths: row (t, hq) of token i of sequence b over that
 * sequence's packed keys. With causal != 0 it sees key j iff j <= i + len_b - n_b (n_b tokens,
 * len_b keys: a prompt where they are equal, a chunk behind earlier keys otherwise), else all.
 * A row that sees no key is 0.
 *   q, o     : [T][Hq][D] bf16, o may be q;  k, v : [Tk][Hkv][D] bf16.
 *   starts   : [B + 1] int32, the sequences' rows of q.
 *   k_starts : [B + 1] int32, their rows of k and v.
 *   workspace : ef_attention_packed_workspace_size(...) bytes, 16-byte aligned (may be NULL where
 *              that is 0); one for larger T, Tk and B serves smaller ones. It holds partial states
 *              where few rows have many keys, behind the counter region of ef_attention_splitkv's
 *              workspace, which is not touched: one workspace serves both. Calls that overlap in
 *              time must not share one.
 * Limit beside those of the other calls: T Hq / 128 + B Hkv <= 2^23 (workgroups of a launch, partial
 * states among them).
 */
ef_status ef_attention_packed(const void* q, const void* k, const void* v, const int* starts,
                              const int* k_starts, void* o, int T, int Tk, int B, int Hq, int Hkv,
                              int D, float scale, int causal, void* workspace,
                              size_t workspace_bytes, void* stream);

/* Workspace bytes of ef_attention_packed; 0 for invalid arguments too. */
size_t ef_attention_packed_workspace_size(int T, int Tk, int B, int Hq, int Hkv, int D);

#ifdef __cplusplus
}
#endif

#endif /* EF_ATTENTION_H */
