/*
 * nlb.h -- C ABI of the MI355X (gfx950) implementation of NLB forward recent
 * sampling: per-node fixed-size hash tables of down-sampled temporal
 * neighbours, maintained on the GPU batch by batch, and batched queries that
 * gather the stored neighbours with their features and a cosine time
 * encoding.
 *
 * Method: Luo & Li, "Scalable and Efficient Temporal Graph Representation
 * Learning via Forward Recent Sampling", arXiv 2402.01964.
 *   - Sec. 3, Def. "Temporal network": a time-ordered stream of undirected
 *     links (u, v, t).  Here link i of the stream gets the 0-based arrival
 *     index e = i (its "edge id"); later means larger e.
 *   - Sec. 3, eq. (1): the temporal neighbours of u at time t are links of u
 *     with timestamp t' < t (strict).
 *   - Sec. 4.2: table S_u has s slots.  Link (u, v, t) offers (v, t, e) to
 *     S_u at slot hash(v, t) and (u, t, e) to S_v at slot hash(u, t), with
 *     hash(v, t) = (q1*v + q2*t) mod s (NLB-edge, eq. (2)) or
 *     hash(v) = q1*v mod s (NLB-node, eq. (3)).  An empty slot takes the
 *     offer; an occupied slot is replaced with probability alpha.  Tables are
 *     updated after the current batch's queries are answered.
 *   - Sec. 4.4: a query (u, t) retrieves S_u^t: each neighbour's status
 *     (node feature row), the link's features and the encoded time.
 *   - App. C: the time encoding is a vector of cosines of w_k * dt + b_k
 *     (the paper's [cos, sin] pairs are the case b_k in {0, -pi/2}).
 *
 * Random draws.  The replacement coin of the offer of link e to its first
 * endpoint (k = 0, table of src) or second endpoint (k = 1, table of dst) is
 * the high 32 bits of output number 2e+k+1 of SplitMix64 (Steele, Lea &
 * Flood, OOPSLA 2014) started from state `seed`.  The offer replaces an
 * occupied slot iff coin < floor(alpha * 2^32) (always when alpha = 1).  The
 * result of every call is therefore a deterministic function of the stream,
 * the parameters and the seed, and equals inserting the links one at a time
 * in stream order, whatever the batch sizes.
 *
 * Conventions for every entry point:
 *   - Pointers named "device" are HIP device memory on the table's device;
 *     the library never frees or retains them beyond what is stated.
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *     Calls are asynchronous and ordered on that stream; use one stream (or
 *     order streams yourself) per table.
 *   - Return value: NLB_OK or an NLB_E* code.  Argument errors are detected
 *     on the host before anything is enqueued and leave the table unchanged.
 *     Errors found by kernels (out-of-range node ids, timestamps >= 2^30 or
 *     out of order) are recorded on the device and reported by nlb_status.
 *   - A table is used from one host thread at a time.  Distinct tables are
 *     independent.  No C++ exception crosses this interface.
 */
#ifndef NLB_H
#define NLB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Return codes. */
#define NLB_OK 0
#define NLB_EINVAL 1   /* bad argument (NULL pointer, size or parameter out of range) */
#define NLB_ENOMEM 2   /* device allocation failed */
#define NLB_EDEVICE 3  /* no usable GPU, or a HIP call failed */
#define NLB_EORDER 4   /* (nlb_status) timestamps decreased, or a timestamp >= 2^30 */
#define NLB_ERANGE 5   /* node id outside [0, num_nodes), or more than 2^32-1 links */
#define NLB_ESCRATCH 6 /* nlb_rnn_update_noalloc: the call needs more working memory than the
                          library's static array holds */

/* Key choice of Sec. 4.2. */
#define NLB_KEY_EDGE 0 /* key (neighbour, time): slot by eq. (2) */
#define NLB_KEY_NODE 1 /* key neighbour: slot by eq. (3) */

#define NLB_MAX_SLOTS 1024

typedef struct nlb_table nlb_table;

typedef struct nlb_config {
    int64_t num_nodes;      /* N: node ids are 0..N-1; 1 <= N <= 2^31-1 */
    int32_t s;              /* slots per node, 1..NLB_MAX_SLOTS */
    int32_t key_mode;       /* NLB_KEY_EDGE or NLB_KEY_NODE */
    double alpha;           /* replacement probability, 0 < alpha <= 1 */
    uint64_t seed;          /* start state of the coin generator */
    uint64_t q1, q2;        /* hash primes of eq. (2)/(3); 0 selects 1000000007 / 998244353;
                               each must be < 2^31 */
    int32_t d_time;         /* time-encoding width; 0 = no time encoding */
    const float *time_w;    /* device fp32[d_time] frequencies, borrowed for the table's life */
    const float *time_b;    /* device fp32[d_time] phases, borrowed for the table's life */
    const void *edge_feat;  /* device [edge_rows][edge_row_bytes] link features indexed by
                               arrival index, borrowed; NULL = none */
    int64_t edge_rows;      /* rows of edge_feat; a stored link with e >= edge_rows gathers zeros */
    int32_t edge_row_bytes; /* bytes per link-feature row, a multiple of 4 (0 with NULL) */
    const void *node_feat;  /* device [num_nodes][node_row_bytes] node rows, borrowed; NULL = none */
    int32_t node_row_bytes; /* bytes per node row, a multiple of 4 (0 with NULL) */
    int32_t device;         /* HIP device ordinal that holds the table; -1 = current device */
} nlb_config;

/* Output buffers of nlb_sample (device pointers, row-major, in slot order).
 * Any member may be NULL to skip that output.  For query i and slot a:
 *   nbr  int32 [nq][s]                  stored neighbour id, -1 if not valid
 *   eid  uint32[nq][s]                  stored arrival index, 0xFFFFFFFF if not valid
 *   ts   uint32[nq][s]                  stored timestamp t', 0xFFFFFFFF if not valid
 *   tenc fp32  [nq][s][d_time]          cos(fmaf(w_k, (float)(tq - t'), b_k)), 0 if not valid
 *   efeat bytes[nq][s][edge_row_bytes]  edge_feat row eid, zero bytes if not valid
 *   nfeat bytes[nq][s][node_row_bytes]  node_feat row nbr, zero bytes if not valid
 *   self  bytes[nq][node_row_bytes]     node_feat row of the query node (zeros if the id is
 *                                       out of range)
 * A slot is valid when it is non-empty and its timestamp t' < tq (eq. (1)).
 * tenc is within 1e-5 absolute of the cosine, taken in double, of the fp32
 * argument fmaf(w_k, (float)(tq - t'), b_k); everything else is exact. */
typedef struct nlb_sample_out {
    int32_t *nbr;
    uint32_t *eid;
    uint32_t *ts;
    float *tenc;
    void *efeat;
    void *nfeat;
    void *self;
} nlb_sample_out;

typedef struct nlb_info {
    int64_t num_nodes;
    int32_t s;
    int32_t key_mode;
    uint64_t threshold;     /* floor(alpha * 2^32), or 2^32 for alpha == 1 */
    uint64_t q1, q2;
    uint64_t interactions;  /* links inserted so far = arrival index of the next link, as
                               counted by eager calls; nlb_status refreshes it from the
                               device count, which also counts graph replays */
    int64_t table_bytes;    /* device bytes owned by the table */
    int32_t block_bytes;    /* bytes of one node's slot block */
    int32_t device;
    int32_t rnn_form;       /* GRU pass of the last nlb_rnn_update: NLB_RNN_FORM_* */
} nlb_info;

/* Forms of the GRU pass of nlb_rnn_update: none run yet; tiles of listed
 * rows with the weights streamed from L2; the weight-stationary form (the
 * weights held in registers for the whole launch, one workgroup per CU),
 * used when the statuses have 16-byte rows, pad32(d) <= 128 and
 * pad32(d) + pad32(d) + pad32(d_time) + pad32(edge_dim) <= 384. */
#define NLB_RNN_FORM_NONE 0
#define NLB_RNN_FORM_TILED 1
#define NLB_RNN_FORM_WEIGHT_STATIONARY 2

/* Create an empty table (Sec. 4.2: fixed-size GPU memory of s slots per
 * node, all empty).  Validates `cfg`, allocates and zeroes the slot blocks on
 * cfg->device, and stores *out only on success.  Errors: NLB_EINVAL (NULL
 * argument, parameter out of range, row bytes not a multiple of 4, feature
 * pointer and row bytes disagreeing), NLB_EDEVICE (no GPU), NLB_ENOMEM. */
int nlb_create(const nlb_config *cfg, nlb_table **out);

/* Insert the n links (src[i], dst[i], t[i]), i < n, as links
 * interactions..interactions+n-1 of the stream (Sec. 4.2).  src, dst, t are
 * device arrays of n elements, read during the call's kernels.  Each link
 * offers to both endpoint tables; conflicts inside the batch resolve exactly
 * as sequential insertion would.  Timestamps must be < 2^30 and
 * non-decreasing across calls; node ids must be in [0, N).  Links with an
 * out-of-range endpoint or timestamp are skipped and flagged for
 * nlb_status, but still consume their arrival index.  n == 0 is a no-op.
 * Errors: NLB_EINVAL (NULL table or array with n > 0; n >= 2^31),
 * NLB_ERANGE (the arrival index would exceed 2^32-2), NLB_EDEVICE (launch
 * failure).  The kernels take the batch's arrival indices from a link count
 * kept on the device and advance it (the host keeps its own count for the
 * NLB_ERANGE test and nlb_get_info), so the call may be captured in a HIP
 * graph: every replay inserts its links as the next links of the stream
 * (a replay that would pass 2^32 - 1 links is skipped and flagged for
 * nlb_status as NLB_ERANGE). */
int nlb_insert_batch(nlb_table *h, const int32_t *src, const int32_t *dst,
                     const uint32_t *t, uint32_t n, void *stream);

/* Answer nq queries (node[i], tq[i]) from the tables as they stand after the
 * inserts enqueued before this call (Sec. 4.4 retrieval; eq. (1) strict
 * mask; App. C time encoding).  node and tq are device arrays of nq
 * elements; out holds device output pointers as described above and is read
 * during the call only.  A query node outside [0, N) yields an all-invalid
 * answer and is flagged for nlb_status.  nq == 0 is a no-op.
 * Errors: NLB_EINVAL (NULL table, out or array with nq > 0; tenc/efeat/nfeat/
 * self requested without the matching configuration), NLB_EDEVICE.
 * The call only enqueues kernels (no allocation, memset or synchronisation):
 * it may be captured in a HIP graph and replayed on the same buffers. */
int nlb_sample(nlb_table *h, const int32_t *node, const uint32_t *tq, uint32_t nq,
               const nlb_sample_out *out, void *stream);

/* Second-hop retrieval (Sec. 4.4: if v is stored in S_u^t, S_v^t holds
 * down-sampled second-hop neighbours of u).  hop1_nbr is the device nbr
 * output [nq][s] of an nlb_sample call for queries (node[i], tq[i]); tq is
 * the same device array of nq query times.  For every first-hop entry
 * (i, a) with neighbour v = hop1_nbr[i*s + a], the call answers the query
 * (v, tq[i]) exactly as nlb_sample would, into row i*s + a of each output:
 * nbr/eid/ts [nq][s][s], tenc [nq][s][s][d_time], efeat/nfeat
 * [nq][s][s][row bytes], self [nq][s][node_row_bytes] (v's node row).  An
 * empty first-hop entry (v < 0) gives an all-invalid answer and a zero self
 * row without an error; v >= N is flagged as in nlb_sample.  nq*s must be
 * below 2^32.  nq == 0 is a no-op.  Errors: as nlb_sample.  Graph capture:
 * as nlb_sample. */
int nlb_sample_hop2(nlb_table *h, const int32_t *hop1_nbr, const uint32_t *tq, uint32_t nq,
                    const nlb_sample_out *out, void *stream);

/* Time encoding (App. C) of an nlb_sample answer from its timestamp output:
 *   tenc[i][a][k] = cos(fmaf(w_k, (float)(tq[i] - ts[i*s + a]), b_k)),
 *   0 where ts[i*s + a] == 0xFFFFFFFF (an invalid slot),
 * the values nlb_sample writes to its own tenc output, to the same bits.
 * With it a caller splits a retrieval into its table reads (nlb_sample with
 * out->tenc NULL and out->ts set) and the encoding, and runs the encoding on
 * a second stream, ordered after the sample by an event the caller records:
 * the encoding reads neither the tables nor the feature rows, so it may run
 * beside the next nlb_insert_batch.  ts: device uint32 [nq][s] (an nlb_sample
 * ts output); tq: the device array of the nq query times of that call; tenc:
 * device fp32 [nq][s][d_time].  All three are read or written during the
 * call's kernels only and must be 4-byte aligned (16-byte aligned output
 * and d_time % 4 == 0 take the vector form).  nq == 0 is a no-op.
 * Errors: NLB_EINVAL (NULL table or array with nq > 0, a table without a time
 * encoding, misaligned arrays), NLB_EDEVICE.  Graph capture: as nlb_sample. */
int nlb_time_encode(nlb_table *h, const uint32_t *ts, const uint32_t *tq, uint32_t nq, float *tenc,
                    void *stream);

/* Attention aggregation of eq. (4) (Sec. 4.4), forward:
 *   Z_u = MLP_out(r_u, sum_i alpha_i MLP_in(r_v, e, t')),
 *   {alpha_i} = softmax({w^T MLP_in(r_v, e, t')}) over the valid slots of S_u^t,
 * with MLP(x) = W_b ReLU(W_a x + b_a) + b_b, hidden and output width
 * NLB_AGG_HIDDEN.  The neighbour status r_v is its node-feature row, e the
 * stored link's feature row, t' enters through the table's time encoding of
 * tq - t' (as in nlb_sample) and r_u is the query node's row; tables
 * without node or link features contribute no such inputs.  A query with no
 * valid slot aggregates the zero vector; a query node outside [0, N) is
 * flagged for nlb_status and treated as having no slots and a zero row.
 * Weight matrices are bf16 (device, row-major [H][K], each input segment
 * zero-padded to a multiple of 32 columns, rows 16-byte aligned):
 *   w1: [H][pad32(node_dim) + pad32(edge_dim) + pad32(d_time)]  (r_v | e | T-enc)
 *   w2: [H][H];  w3: [H][pad32(node_dim) + H]  (r_u | aggregate);  w4: [H][H]
 * with node_dim / edge_dim the table's row bytes divided by the element size
 * of node_dtype / edge_dtype.  Biases and att (the attention vector w) are
 * device fp32 [H].  All are read during the call only.  Activations are kept
 * in fp32 and fed to bf16 matrix cores as a pair of bf16 terms (hi + lo,
 * relative error 2^-18), accumulating in fp32 over at most ~400 terms
 * (relative error ~2.5e-5 of the sum of magnitudes); through four layers and
 * the softmax, Z is within 2e-4 * (|Z| + the root mean square of Z over the
 * launch) of the same function evaluated in double (measured: <= 3.9e-5).
 * MLP_in's second layer is affine, so the library may apply it once to the
 * softmax-weighted sum of the first layer's outputs instead of to every
 * slot (the logits then use W_b^T w); only the rounding order differs.
 * Attention heads (the experiments use two, App. E): with heads = A, MLP_in's
 * H outputs are split into A consecutive slices of H / A; head a scores a
 * slot with w[slice a] . MLP_in(...)[slice a], takes its own softmax over the
 * valid slots and fills slice a of the aggregate.  A = 1 is the formula
 * above.  One or two heads run in every kernel form, four and eight in the
 * tiled form (tables of at most 64 slots); any other count is NLB_EINVAL.
 * z is device fp32 [nq][H].  Tables with s > 64 are supported for the input
 * shapes the per-query kernel is built for and rejected (NLB_EINVAL) for
 * others: a time encoding of 97 to 128 dimensions with 16-byte-aligned bf16
 * node rows of 97 to 128 values and no link rows or such bf16 link rows, or
 * no node rows and fp32 link rows of 97 to 128 or 161 to 192 values
 * (16-byte aligned) or bf16 link rows of 161 to 192 values (4-byte aligned).
 * nq == 0 is a no-op.  Errors: as nlb_sample, and NLB_EINVAL
 * for a bad weight set.  Graph capture: as nlb_sample (besides its kernels
 * the call makes only host-side attribute queries and settings). */
#define NLB_AGG_HIDDEN 64
#define NLB_DTYPE_F32 0
#define NLB_DTYPE_BF16 1

typedef struct nlb_agg_weights {
    int32_t hidden;          /* must be NLB_AGG_HIDDEN */
    int32_t node_dtype;      /* element type of the table's node rows: NLB_DTYPE_F32 / _BF16 */
    int32_t edge_dtype;      /* element type of the table's link rows */
    int32_t heads;           /* attention heads A: 0 or 1 for one, else 2, 4 or 8 */
    const uint16_t *w1;      /* bf16 bits */
    const float *b1;
    const uint16_t *w2;
    const float *b2;
    const float *att;
    const uint16_t *w3;
    const float *b3;
    const uint16_t *w4;
    const float *b4;
} nlb_agg_weights;

int nlb_aggregate(nlb_table *h, const int32_t *node, const uint32_t *tq, uint32_t nq,
                  const nlb_agg_weights *wts, float *z, void *stream);

/* Node-status update of Sec. 4.4: after a link (u, v, t) with features e,
 * r_u <- RNN([r_u, r_v, t, e]) and r_v <- RNN([r_v, r_u, t, e]), for a batch
 * of n links (src, dst, t: device arrays of n elements) whose link-feature
 * rows are first_eid .. first_eid + n - 1 of the table's link rows (rows at
 * or past edge_rows read as zeros); first_eid = NLB_EID_LAST_BATCH takes the
 * arrival indices of the n links inserted last (the table's device link
 * count when the update runs, minus n), as a step that inserts a batch and
 * then updates the statuses needs, also when replayed from a HIP graph.
 * The RNN is a GRU cell with input x = [r_other ; T-enc(t) ; e] and hidden
 * state h = r_self:
 *   r = sigmoid(W_ir x + b_ir + W_hr h + b_hr)
 *   z = sigmoid(W_iz x + b_iz + W_hz h + b_hz)
 *   n = tanh(W_in x + b_in + r * (W_hn h + b_hn))
 *   h' = (1 - z) n + z h
 * with T-enc(t) the table's time encoding cos(w_k t + b_k) of the link time
 * (argument fmaf(w_k, (float)t, b_k)).  Batch semantics: every update reads
 * the statuses as they were before the call, and a node that several links
 * of the batch touch takes the update of the latest one (larger index; on a
 * self-loop the dst side's).  status is a device array [N][status_dim] of
 * status_dtype elements, updated in place (it may be the table's node_feat
 * buffer, so later queries gather the new statuses); rows of nodes that no
 * link touches are not written.  A link with an endpoint outside [0, N) is
 * skipped and flagged for nlb_status.  Weights (device, read during the
 * call, bf16 rows 16-byte aligned, each input segment zero-padded to a
 * multiple of 32 columns, gate rows in the order r | z | n):
 *   w_ih: [3 d][pad32(d) + pad32(d_time) + pad32(edge_dim)]  (r_other | T-enc | e)
 *   w_hh: [3 d][pad32(d)];  b_ih, b_hh: fp32 [3 d]
 * with d = status_dim and edge_dim the table's link row bytes over the size
 * of edge_dtype.  Numerics: fp32 activations enter bf16 matrix cores as
 * hi + lo pairs (2^-18 relative), bf16 ones as one term, with fp32
 * accumulation; an fp32 status is within 1e-4 of the same cell evaluated in
 * double, a bf16 one within one bf16 rounding of it.  Calls on one table
 * must be ordered (same stream): they share the table's working buffers,
 * which the first call (and a larger batch) allocates.  n == 0 is a no-op.
 * Graph capture: a call that allocates (see above) must not be captured;
 * once an earlier call on the table has sized the working memory for at
 * least n links, the call only enqueues kernels and may be captured and
 * replayed (no call number or host-side state is involved; with
 * first_eid = NLB_EID_LAST_BATCH it follows the inserts replayed before it).
 * Errors: NLB_EINVAL (NULL table, weights or array with n > 0; n >= 2^31;
 * bad dtype or dimension; misaligned pointers; a 16-row tile that does not
 * fit the LDS), NLB_ENOMEM, NLB_EDEVICE. */
#define NLB_RNN_MAX_DIM 1024
#define NLB_EID_LAST_BATCH UINT64_MAX

typedef struct nlb_gru_weights {
    int32_t status_dim;      /* d, 1 .. NLB_RNN_MAX_DIM */
    int32_t status_dtype;    /* NLB_DTYPE_F32 / _BF16 */
    int32_t edge_dtype;      /* element type of the table's link rows */
    const uint16_t *w_ih;    /* bf16 bits */
    const uint16_t *w_hh;
    const float *b_ih;
    const float *b_hh;
} nlb_gru_weights;

int nlb_rnn_update(nlb_table *h, const int32_t *src, const int32_t *dst, const uint32_t *t, uint32_t n,
                   uint64_t first_eid, const nlb_gru_weights *wts, void *status, void *stream);

/* nlb_rnn_update for callers that cannot allocate device memory: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments, kernels and results; it allocates and frees nothing
 * (device memory, host-pinned memory or library workspaces) and sets no
 * memory with hipMemset: its working memory -- the winner word of each of
 * the table's N nodes (8 B), a list of 16 B per pair row, the GRU weights
 * repacked in matrix-operand fragments (3 KiB per 16 status columns and
 * 32 input columns of w_ih and w_hh together), and 2 n staged status rows
 * -- lives in one static device array of NLB_NOALLOC_SCRATCH bytes per
 * device, which the library holds until the process ends.  The call needs
 * align256(8 N) + align256(16 (2 n) + 256) + align256(3072 (pad32(d) / 16)
 * ((k_x + pad32(d)) / 32)) + 2 n * status row bytes of it (k_x: the row
 * width of w_ih), and returns NLB_ESCRATCH when that exceeds the array
 * (nothing is enqueued then).  Every call on a device shares that device's
 * array: the call clears what it needs cleared (the winner words, with a
 * fill kernel) and keeps no state across calls, but calls that overlap in
 * time on one device -- other streams, other threads, other tables -- race
 * and must be ordered by the caller.  Besides the NLB_ESCRATCH case, errors
 * are those of nlb_rnn_update.  The first call on a device looks up the
 * array's device address (hipGetSymbolAddress) with that device current. */
#define NLB_NOALLOC_SCRATCH (64u << 20)

int nlb_rnn_update_noalloc(nlb_table *h, const int32_t *src, const int32_t *dst, const uint32_t *t,
                           uint32_t n, uint64_t first_eid, const nlb_gru_weights *wts, void *status,
                           void *stream);

/* Softmax attention over packed sequences, with a learned bias on the gap
 * between two positions: the layer that reads retrieved lists (nlb_sample's
 * answers) or whole histories.  For query row i and key row j of one sequence
 * and query head h, which reads key/value head h / (heads / kv_heads):
 *   s_ij = scale q_i . k_j + bias[bucket(pos_i - pos_j)][h]
 *   o_i  = sum_j softmax_j(s_i) v_j,   lse_i = log sum_j exp(s_ij)
 * over the keys open to row i.  A row without an open key has o_i = 0 and
 * lse_i = -infinity.
 *   Sequences.  Sequence b has the query rows q_start[b] .. q_start[b + 1] - 1
 * and the key rows k_start[b] .. k_start[b + 1] - 1 (device int32 [batch + 1],
 * non-decreasing; the host need not know the lengths, which may be zero).
 * q_start NULL: q_rows / batch rows each; k_start NULL: k_rows / batch keys
 * each (the division must leave no rest).  Rows before the first and behind
 * the last sequence are neither read nor written.  Starts outside [0, rows]
 * are taken as the nearest end, so no call reads or writes outside its rows.
 * With q_start NULL and q_rows == batch (a retrieved list per query, or one
 * new token per sequence) the call runs in a form made for single rows.  The
 * host sees the average length only: of lists of 64 keys or fewer on average
 * (8192 and more, times key/value heads; the gradients' lists likewise) each is
 * one lane group's, however long, and the call waits for the longest (10 000
 * lists of 30 keys, one of them of 10 000: 3.6 ms and 12 for the gradients,
 * where it has 30 too 0.03 and 0.07).  With q_start given, 0 .. batch, single
 * rows take the form for rows of any number instead (0.3 and 1.0 ms; 0.17 and
 * 0.7 for short lists).
 *   Rows.  q, o: [q_rows][heads][dim], k, v: [k_rows][kv_heads][dim], of type
 * dtype, at any row and head strides (in values, 0 .. 2^31 - 1); a row's dim
 * values are contiguous, so slices of a joint projection need no copy.
 * Written rows must not overlap each other or what the call reads.
 *   Open keys.  causal = 1: key j is open to row i if j <= i + lk - lq (i, j
 * counted in the sequence, lq and lk its lengths): the last query row stands
 * at the last key row.  k_pos (device uint32 [k_rows] or NULL): rows with
 * k_pos = 0xFFFFFFFF are closed to every query, as nlb_sample's ts marks empty
 * slots; what their k and v hold is not used.  A key that causal closes to
 * some rows only must hold finite values, or those rows may become NaN.
 *   scale: 0, or of a magnitude from 2^-20 to 2^20.
 *   Bias.  buckets = 0: none (bias NULL).  Else bias is a device array
 * [buckets][heads] of dtype, bounds a device int32 [buckets - 1], none
 * below the one before it, and bucket(x) the number of bounds <= x.  Positions
 * are q_pos (device uint32 [q_rows]) and k_pos, whose difference is clamped to
 * int32 (as nlb_sample's tq and ts go in), or without either the places
 * i + lk - lq and j.  A bias at or below -2^100 closes its bucket; any other
 * beyond 2^20 in magnitude counts as 2^20 (with its sign): a mask of -1e9 takes
 * all weight from its keys, and a row that has no other keys spreads it over
 * them by their scores.
 *   Numerics.  Sums, the softmax's maximum and sum, and lse are fp32.  bf16
 * rows: products of bf16 values are exact in fp32, softmax weights enter the
 * second product as bf16 (in the single-row form as fp32), o is rounded once.
 * fp32 rows: fp32 products throughout.  Scores are fp32 too: where a row's
 * scores reach a magnitude of x, its weights (and what the backward pass makes
 * of lse) are off by some 2^-22 x of themselves.  The same call gives the same
 * bits.
 *   Working memory: nlb_attention_work bytes of device memory (16-byte
 * aligned, may be NULL if that is 0), used by the call's kernels only; calls
 * that may overlap in time need one each.  lse (device fp32 [q_rows][heads])
 * may be NULL where no backward pass follows.  Only enqueues kernels: may be
 * captured in a HIP graph.  No table is involved; device names the device of
 * the arrays and the stream (-1: the current one).  Errors: NLB_EINVAL (as
 * above; more than 2^31 - 1024 rows; more than 2^31 - 1 workgroups, of which
 * a head takes one for each sequence and each 32 or 128 rows),
 * NLB_ESCRATCH (work_bytes too few), NLB_EDEVICE. */
#define NLB_ATT_MAX_DIM 128
#define NLB_ATT_MAX_HEADS 256
#define NLB_ATT_MAX_BUCKETS 64

typedef struct nlb_att_rows {
    void *data;
    int64_t row_stride, head_stride;   /* values */
} nlb_att_rows;

typedef struct nlb_att_call {
    int32_t device;          /* HIP device ordinal, -1 = current */
    int32_t dtype;           /* NLB_DTYPE_F32 / _BF16: q, k, v, o, bias and their gradients */
    int32_t heads, kv_heads; /* heads a multiple of kv_heads, at most NLB_ATT_MAX_HEADS */
    int32_t dim;             /* 1 .. NLB_ATT_MAX_DIM */
    int32_t causal;          /* 0 or 1 */
    int32_t buckets;         /* 0 .. NLB_ATT_MAX_BUCKETS */
    float scale;
    uint32_t batch, q_rows, k_rows;
    const int32_t *q_start, *k_start;
    const void *bias;
    const int32_t *bounds;
    const uint32_t *q_pos, *k_pos;
    nlb_att_rows q, k, v;    /* not written */
} nlb_att_call;

/* Device bytes that nlb_attention (backward = 0) or nlb_attention_backward
 * (1) of this call works in; a host computation.  Errors: NLB_EINVAL. */
int nlb_attention_work(const nlb_att_call *call, int32_t backward, size_t *bytes);

int nlb_attention(const nlb_att_call *call, const nlb_att_rows *o, float *lse, void *work, size_t work_bytes,
                  void *stream);

/* Gradients of nlb_attention: from the same call (its sequences, positions and
 * bias unchanged), its outputs o and lse, and the gradient dout of o (rows as
 * o), with p_ij = exp(s_ij - lse_i):
 *   ds_ij = p_ij (dout_i . v_j - D_i),   D_i = sum_j p_ij dout_i . v_j
 *   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij dout_i
 *   dbias[b][h] = the sum of ds_ij over the pairs of bucket b
 * dk and dv sum over the query heads of a key/value head.  All rows of the
 * sequences are written (zeros for closed keys and for rows without open
 * keys), rows outside them are not.  q and dout hold finite values in all rows
 * of the sequences, those without open keys too.  dbias: device
 * [buckets][heads] of dtype, or NULL where it is not wanted.
 *   Single rows have a form of their own here where they are lists: at most 4
 * query heads on a key/value head, and up to 64 keys a list on average (up to
 * 1024 for 8192 lists times key/value heads and more).  All other calls, single
 * rows over longer histories and larger groups of heads among them, take the
 * form for rows of any number: right, but slow for single rows (200 000 lists
 * of 10 bf16 rows, 8 heads on one: 33 ms; 4 heads on one: 0.6).
 *   Numerics.  As nlb_attention; in the form for rows of any number softmax
 * weights and ds enter the second products as bf16 for bf16 rows, in that for
 * lists as fp32.  D_i: in the form for lists its own sum (o is not read); else
 * dout . o, corrected by a pass over the keys for bf16 rows, and for fp32 rows
 * where dbias is wanted.  dbias sums ds in fp32 and fp64, rounded once.  No
 * atomics on results: the same call gives the same bits.
 *   Work, capture and errors: as nlb_attention (NLB_EINVAL also for dbias
 * without buckets).  dbias takes 4 heads x buckets bytes for each sequence and
 * each 32 or 128 query rows (in the form for lists, of 2048 workgroups at most). */
int nlb_attention_backward(const nlb_att_call *call, const nlb_att_rows *o, const float *lse,
                           const nlb_att_rows *dout, const nlb_att_rows *dq, const nlb_att_rows *dk,
                           const nlb_att_rows *dv, void *dbias, void *work, size_t work_bytes, void *stream);

/* Layer norm of rows, before and after such a layer:
 *   mean = sum x / width,  rstd = (sum (x - mean)^2 / width + eps)^-1/2
 *   y = (x - mean) rstd w + b
 * x, y: device rows of `width` contiguous values of dtype, x_stride and
 * y_stride values apart (0 .. 2^31 - 1; y may be x).  w, b: device fp32
 * [width], NULL for ones and zeros.  mean, rstd: device fp32 [rows], written
 * (NULL where no backward pass follows).  All sums are fp32, each row's values
 * are read once; y is rounded once.  rows = 0 is a no-op.
 *   nlb_layer_norm_backward, from the same call with mean and rstd as written,
 * and the gradient dy of y:
 *   g = dy w,  xh = (x - mean) rstd
 *   dx = rstd (g - sum g / width - xh sum (g xh) / width)
 *   dw = sum over rows of dy xh,  db = sum over rows of dy
 * dx may be dy.  dw, db: device fp32 [width], written (not added to), either
 * may be NULL; with both NULL no work is needed, else nlb_layer_norm_work
 * bytes of device memory (16-byte aligned) that the call's kernels use.  Sums
 * over rows are fp32 within a workgroup, then fp64, in a fixed order.
 *   Only enqueues kernels: may be captured in a HIP graph.  Errors: NLB_EINVAL
 * (NULL rows, mean or rstd, a bad size, type, stride, alignment or eps),
 * NLB_ESCRATCH, NLB_EDEVICE. */
#define NLB_NORM_MAX_WIDTH 8192

typedef struct nlb_norm_call {
    int32_t device;          /* HIP device ordinal, -1 = current */
    int32_t dtype;           /* NLB_DTYPE_F32 / _BF16: x, y, dy, dx */
    uint32_t rows;
    int32_t width;           /* 1 .. NLB_NORM_MAX_WIDTH */
    const void *x;
    int64_t x_stride;        /* values */
    const float *w;
    float *mean, *rstd;
} nlb_norm_call;

int nlb_layer_norm(const nlb_norm_call *call, const float *b, float eps, void *y, int64_t y_stride, void *stream);

int nlb_layer_norm_work(const nlb_norm_call *call, size_t *bytes);

int nlb_layer_norm_backward(const nlb_norm_call *call, const void *dy, int64_t dy_stride, void *dx,
                            int64_t dx_stride, float *dw, float *db, void *work, size_t work_bytes, void *stream);

/* Rows of a learned table by id, and the table's gradient: the rows that
 * nlb_sample gathers as nfeat and self are those of its nbr and node ids, so
 * that a table can be trained through them.
 *   nlb_lookup: out_i = scale table[ids[i]], zeros where ids[i] is none of 0 ..
 * rows - 1 (nbr's -1, an empty slot).  table: device [rows][width], out: device
 * [n][width] of dtype, at any row stride (in values, 0 .. 2^31 - 1); a row's
 * values are contiguous.  Rounded once.
 *   nlb_lookup_backward, from the same call and the gradient dout of out:
 *   dtable_r = scale (sum of dout_i over the i with ids[i] = r)
 * list and count NULL: the whole gradient, [rows][width], zeros for rows that
 * do not occur.  Else the rows that occur: list (device int32 [n]) gets their
 * ids, ascending, and -1 behind them, count (device uint32) their number, and
 * the first `count` rows of dtable ([n][width]) their gradients; the rows behind
 * them stay as they are.  The ids are sorted; a row's gradients are added up in
 * fp32 in an order that the ids, n, the width and the type set, no atomics on
 * results: the same call gives the same bits, but a popular row's columns may
 * differ in their last bits from those of a wider call.  Rows of ids outside the
 * table are not read.
 *   Work: nlb_lookup_work bytes of device memory (16-byte aligned; listed = 0
 * for the whole gradient, 1 for the rows that occur), used by the call's kernels
 * only.  Only enqueues kernels: may be captured in a HIP graph.  Written rows
 * must not overlap each other or what is read.  Errors: NLB_EINVAL,
 * NLB_ESCRATCH, NLB_EDEVICE. */
#define NLB_LOOKUP_MAX_WIDTH 65536

typedef struct nlb_lookup_call {
    int32_t device;          /* HIP device ordinal, -1 = current */
    int32_t dtype;           /* NLB_DTYPE_F32 / _BF16: table, out and their gradients */
    uint32_t n, rows;        /* ids (0 .. 2^31 - 1); rows of the table (1 .. 2^31 - 1) */
    int32_t width;           /* 1 .. NLB_LOOKUP_MAX_WIDTH */
    float scale;             /* finite */
    const int32_t *ids;
} nlb_lookup_call;

int nlb_lookup(const nlb_lookup_call *call, const void *table, int64_t table_stride, void *out, int64_t out_stride,
               void *stream);

int nlb_lookup_work(const nlb_lookup_call *call, int32_t listed, size_t *bytes);

int nlb_lookup_backward(const nlb_lookup_call *call, const void *dout, int64_t dout_stride, void *dtable,
                        int64_t dtable_stride, int32_t *list, uint32_t *count, void *work, size_t work_bytes,
                        void *stream);

/* RMS norm of each head's queries and keys and their rotation by position, in
 * one pass, between the projections and the attention:
 *   u = x (sum x^2 / dim + eps)^-1/2 w,  a_i = pos freq[i]  for i < m = freqs
 *   y_i = u_i cos a_i - u_{m+i} sin a_i,  y_{m+i} = u_{m+i} cos a_i + u_i sin a_i
 *   y = u  behind the first 2 m values of a head
 * so that the product of a query and a key depends on the gap of their
 * positions alone: by places, or by timestamps with the frequencies of a time
 * encoding (nlb_sample's tq and ts go in as they are).
 *   Rows.  q: [q_rows][heads][dim], k: [k_rows][kv_heads][dim] of dtype, as for
 * nlb_attention, and so the results (which may be q and k themselves); k_rows
 * = 0: no keys.  q_pos, k_pos: device uint32, one for each row (NULL: 0, where
 * freqs is 0).  A row at position 0xFFFFFFFF is an empty slot, as nlb_sample's
 * ts marks it: it is not read, its result and gradient are zeros and it takes
 * no part in dwq and dwk.  freq: device fp32 [freqs]; wq, wk: device fp32 [dim],
 * NULL for ones.
 *   Numerics.  Angles are formed and reduced in 64 bits: their error is some
 * 2^-24 and |a| 2^-51.  Sums and products are fp32, each row's values are read
 * once and rounded once.  The sum of a head's squares has to fit fp32, and its
 * mean and eps have to be 2^-126 or more together (values of 2^60 at most, and
 * of 2^-59 where eps is 0): others have no meaningful result.  With eps = 0 a
 * head of zeros is NaN, as in the formula; an empty slot is zeros all the same.
 *   nlb_norm_rotate_backward, from the same call (q and k as they went in) and
 * the gradients dq_out, dk_out of the results: with du = the gradient rotated
 * by -a, g = du w, r = the norm's factor,
 *   dq = r (g - x r^2 sum(g x) / dim),  dwq = sum over rows and heads of du x r
 * and so for k.  dq, dk may be dq_out, dk_out.  dwq, dwk: device fp32 [dim],
 * written (not added to), each may be NULL; with both NULL no work is needed,
 * else nlb_norm_rotate_work bytes of device memory (16-byte aligned) that the
 * call's kernels use.  Their sums are fp32 within a workgroup, then fp64, in a
 * fixed order: the same call gives the same bits.
 *   Only enqueues kernels: may be captured in a HIP graph.  Written rows must
 * not overlap each other or, but for the arrays named above, what the call
 * reads.  Errors: NLB_EINVAL, NLB_ESCRATCH, NLB_EDEVICE. */
typedef struct nlb_rotate_call {
    int32_t device;          /* HIP device ordinal, -1 = current */
    int32_t dtype;           /* NLB_DTYPE_F32 / _BF16: q, k, the results and their gradients */
    int32_t dim;             /* 1 .. NLB_ATT_MAX_DIM */
    int32_t freqs;           /* 0 .. dim / 2 */
    int32_t heads, kv_heads; /* 1 (kv_heads without keys: 0) .. NLB_ATT_MAX_HEADS */
    uint32_t q_rows, k_rows;
    float eps;
    const float *freq;
    const uint32_t *q_pos, *k_pos;
    const float *wq, *wk;
    nlb_att_rows q, k;       /* not written */
} nlb_rotate_call;

int nlb_norm_rotate(const nlb_rotate_call *call, const nlb_att_rows *q_out, const nlb_att_rows *k_out, void *stream);

int nlb_norm_rotate_work(const nlb_rotate_call *call, size_t *bytes);

int nlb_norm_rotate_backward(const nlb_rotate_call *call, const nlb_att_rows *dq_out, const nlb_att_rows *dk_out,
                             const nlb_att_rows *dq, const nlb_att_rows *dk, float *dwq, float *dwk, void *work,
                             size_t work_bytes, void *stream);

/* A gated linear recurrence over packed sequences, channel by channel: a state
 * for each node's history that a scan makes for all its events at once, or that
 * one event moves on (a sequence of one row).
 *   z_t = sigmoid(g_t),  h_t = z_t h_{t-1} + (1 - z_t) x_t
 * from h0[b] (NULL: zeros) before sequence b's first row; last[b] is the state
 * behind its last row (h0[b] where it has none).
 *   Sequences.  Sequence b has the rows start[b] .. start[b + 1] - 1 (device
 * int32 [batch + 1], non-decreasing; lengths may be zero, the host need not
 * know them).  start NULL: rows / batch rows each (no rest).  Starts outside
 * [0, rows] are taken as the nearest end.  Rows before the first and behind the
 * last sequence are neither read nor written.  The rows set how many workgroups
 * there are, and each passes its share of the sequences without rows on one
 * after the other: where there are many of them beside few rows, they are the
 * call's time (2000 rows of 100 fp32 values in 20 000 sequences: 0.25 ms either
 * pass, in 200 000: 3.3; a call of no rows at all: some 0.5 us a sequence).
 *   Rows.  x, g, h: [rows][width] of dtype, at any row stride (in values,
 * 0 .. 2^31 - 1); a row's values are contiguous.  h may be x.  h0, last: device
 * fp32 [batch][width], contiguous; last may be NULL, and may be h0 where start
 * is NULL and rows == batch (else arrays that overlap are refused).  states
 * (device fp32 [rows / NLB_SCAN_STATE_ROWS, rounded up][width]) is what a
 * backward pass starts from; NULL where none follows.
 *   Numerics.  Gates, states and products are fp32 (1 - z is not formed by
 * subtraction), h is rounded once.  Gates beyond 80 in magnitude count as 80.
 * z and 1 - z are off by at most 12 x 2^-24 of themselves, in calls of bf16 rows
 * by |g| 2^-23 more, which last, states and dh0 have too, fp32 as they are.
 * Maps of some rows each are joined in a fixed tree: the same call gives the
 * same bits.  What one sequence holds (NaN, infinities) does not reach another;
 * behind an infinity a channel's rows of that sequence are infinite or NaN.
 *   nlb_gated_scan_backward, from the same call, states as written, the gradient
 * dh of h and that of last (dlast, NULL: zeros):
 *   d_t = dh_t + z_{t+1} d_{t+1}  (behind the last row: dlast)
 *   dx = (1 - z) d,  dg = z (1 - z) d (h_{t-1} - x),  dh0[b] = z d of the first row
 * (dlast[b] where a sequence has no rows).  h is made again in fp32, not read.
 * dx, dg: rows as x; dx may be dh.  dh0: device fp32 [batch][width] or NULL.
 *   Work: nlb_gated_scan_work bytes of device memory (16-byte aligned, may be
 * NULL if that is 0) for either pass, used by the call's kernels only.  Only
 * enqueues kernels: may be captured in a HIP graph.  Written rows must not
 * overlap each other or, but for the arrays named above, what the call reads.
 * Errors: NLB_EINVAL, NLB_ESCRATCH, NLB_EDEVICE. */
#define NLB_SCAN_MAX_WIDTH 65536
#define NLB_SCAN_MAX_ROWS 2147480000u
#define NLB_SCAN_STATE_ROWS 32

typedef struct nlb_scan_rows {
    void *data;
    int64_t row_stride;      /* values */
} nlb_scan_rows;

typedef struct nlb_scan_call {
    int32_t device;          /* HIP device ordinal, -1 = current */
    int32_t dtype;           /* NLB_DTYPE_F32 / _BF16: x, g, h and their gradients */
    uint32_t rows, batch;
    int32_t width;           /* 1 .. NLB_SCAN_MAX_WIDTH */
    const int32_t *start;
    const float *h0;
    nlb_scan_rows x, g;      /* not written */
} nlb_scan_call;

int nlb_gated_scan_work(const nlb_scan_call *call, size_t *bytes);

int nlb_gated_scan(const nlb_scan_call *call, const nlb_scan_rows *h, float *last, float *states, void *work,
                   size_t work_bytes, void *stream);

int nlb_gated_scan_backward(const nlb_scan_call *call, const float *states, const nlb_scan_rows *dh,
                            const float *dlast, const nlb_scan_rows *dx, const nlb_scan_rows *dg, float *dh0,
                            void *work, size_t work_bytes, void *stream);

/* Free the table's device memory after synchronising its device.  NULL is a
 * no-op.  Borrowed buffers are not touched. */
int nlb_destroy(nlb_table *h);

/* Sizes and counters of a table (host-side values; no synchronisation). */
int nlb_get_info(const nlb_table *h, nlb_info *info);

/* Write the canonical table into device arrays of N*s elements, node-major:
 * nbr (-1 = empty), ts and eid (0xFFFFFFFF = empty).  Ordered on `stream`.
 * For inspection and tests; the layout the kernels use is internal. */
int nlb_export(nlb_table *h, int32_t *nbr, uint32_t *ts, uint32_t *eid, void *stream);

/* Synchronise `stream`, then return and clear the errors kernels recorded
 * since the last call: NLB_OK, NLB_ERANGE (node id out of range, or a
 * replayed insert past 2^32 - 1 links) or NLB_EORDER (timestamp >= 2^30 or
 * decreasing); NLB_ERANGE wins when both.  Also refreshes the link count of
 * nlb_get_info from the device. */
int nlb_status(nlb_table *h, void *stream);

/* Static description of a return code. */
const char *nlb_strerror(int code);

#ifdef __cplusplus
}
#endif

#endif /* NLB_H */
