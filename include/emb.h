/*
 * emb.h -- C ABI of the sparse-embedding hot path on one MI355X (gfx950).
 *
 * The path is one GPU's share of sparse embedding-table training in EmbRace
 * (Li et al., "EmbRace: Accelerating Sparse Communication for Distributed
 * Training of Deep Neural Networks", ICPP '22):
 *
 *   emb_gather             forward lookup of the batch's rows       (Sec. 4.1.1)
 *   emb_grad_coalesce      COALESCE + UNIQUE of the sparse gradient (Sec. 4.2.2,
 *                          Algorithm 1)
 *   emb_pack_by_owner      per-owner send buffers, counts, offsets  (Sec. 4.1.1,
 *                          Sec. 4.1.2: the payload of the gradient AlltoAll)
 *   emb_sparse_adam_apply  row-wise Adam on the rows a shard owns   (Sec. 4.1.1,
 *                          Sec. 5.7)
 *
 * with, around them: the owner-major coalesce that writes the send layout
 * directly, and its prior/delayed split (Algorithm 1); the receiver side of
 * the exchange (a simulated AlltoAll and the merge); the column-wise partition
 * of Sec. 4.1.1 (gradient pack, every owner's lookup, the join of the lookup
 * results); the Table 2 cost model; and a step executor.
 *
 * The dense operators next to the tables in a training step are declared at the
 * end of this file: layer norm of rows (of looked-up rows as well) and the
 * relative position bias by buckets, each with its gradient, AdamW over many
 * tensors, dropout, the norms before and after a block with its gate and
 * residual scale, and the softmax cross entropy over a table's vocabulary.
 *
 * Conventions for every call:
 *  - Array arguments are DEVICE pointers (memory of the current HIP device);
 *    scalars are passed by value.  The caller allocates and owns every buffer;
 *    the calls of the path never allocate, free or keep a pointer after
 *    returning.  The one allocation of the library is the signal memory of
 *    emb_step_signals_create (a few words per handle, kept in a pool for reuse
 *    and never returned to the runtime).
 *  - Tables and gradient rows are dense row-major [rows][D] arrays.  Ids are
 *    int32 row indices in [0, V).
 *  - `stream` is a hipStream_t (NULL: the null stream).  Calls only enqueue
 *    work on it and return without synchronising; outputs are valid once the
 *    stream has reached that point.  Data-dependent sizes (the unique count,
 *    per-owner counts) stay in device memory: later calls read them there, and
 *    grids are sized by the caller's capacity arguments.
 *  - The return value is a host status (EMB_OK or an EMB_ERR_* code).  Argument
 *    errors are found on the host before anything is enqueued.  Errors that
 *    depend on device data (an id or owner out of range) are OR-ed as
 *    EMB_DEV_* flags into *dev_status (an optional int32 in device memory,
 *    NULL to ignore); the caller clears it and reads it after synchronising.
 *  - Calls are reentrant; concurrent calls need distinct outputs and
 *    workspaces.
 */
#ifndef EMB_H
#define EMB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define EMB_ABI_VERSION 3

/* host status codes */
#define EMB_OK 0
#define EMB_ERR_INVALID_ARG 1 /* null pointer, size or range out of bounds */
#define EMB_ERR_WORKSPACE 2   /* workspace smaller than the size query */
#define EMB_ERR_LAUNCH 3      /* the HIP runtime refused a launch */
#define EMB_ERR_UNSUPPORTED 4 /* valid but not supported by this library */

/* gradient element types */
#define EMB_F32 0  /* IEEE binary32 */
#define EMB_BF16 1 /* bfloat16 (upper half of a binary32), widened exactly */

/* device status flags */
#define EMB_DEV_ID_OUT_OF_RANGE 1    /* a token or row id was outside [0, V) */
#define EMB_DEV_OWNER_OUT_OF_RANGE 2 /* row_owner[id] was outside [0, P) */
#define EMB_DEV_STALLED 4            /* internal: a workgroup gave up waiting for the result \
                                        of an earlier one; the outputs are invalid */
#define EMB_DEV_BUCKET_OUT_OF_RANGE 8 /* a pair's entry of bucket_of was num_buckets or more */
#define EMB_DEV_NOT_FINITE 16 /* emb_adamw_step: a moment is infinite or NaN */

int emb_abi_version(void);
const char *emb_status_string(int status);

/*
 * Forward lookup (Sec. 4.1.1: each process looks up its batch in the
 * embedding table).  out[t][j] = table[ids[t]][j] for t < T, j < D: a bit copy.
 *   table [V][D] fp32, ids [T] int32, out [T][D] fp32.
 * An id outside [0, V) yields a zero row and sets EMB_DEV_ID_OUT_OF_RANGE.
 * T == 0 is a no-op.  Requires 1 <= V < 2^31, D >= 1, T >= 0.
 */
int emb_gather(const float *table, int64_t V, int32_t D, const int32_t *ids,
               int32_t T, float *out, int32_t *dev_status, void *stream);

/*
 * COALESCE and UNIQUE of Algorithm 1 (Sec. 4.2.2, "Coalescing Gradients"):
 * the embedding gradient is a sparse COO tensor (Sec. 2.1) with one row per
 * token; rows with the same index are summed into one.
 *   ids [T] int32, grad [T][D] fp32 (EMB_F32) or bf16 (EMB_BF16).
 * Outputs, sized by the capacity T (the unique count U <= T):
 *   uniq_ids    [T]     the U distinct valid ids, ascending
 *   seg_offsets [T + 1] seg_offsets[k] = number of valid tokens whose id is
 *                       below uniq_ids[k]; seg_offsets[U] = valid tokens
 *   uniq_grad   [T][D]  fp32 per-id sums of the gradient rows
 *   num_unique  [1]     U
 * Entries past U are left unspecified.  Tokens with an id outside [0, V) are
 * left out and set EMB_DEV_ID_OUT_OF_RANGE.
 * Sums are accumulated in fp32 in a fixed order that depends only on the ids
 * (sorted position order, in chunks of 32 tokens, then an ordered combine of
 * the chunk partials; a batch of at most 2048 tokens is summed in plain
 * sorted position order): results are bitwise reproducible run to run.
 * In large batches (more than 655360 tokens; more than 131072 where the keys
 * have at most 9 bits) workgroups of one launch hand prefix sums to each other
 * (decoupled look-back); every wait is bounded and a timeout sets
 * EMB_DEV_STALLED.
 * workspace: device memory of at least
 * emb_grad_coalesce_workspace_bytes(T, V, D, grad_dtype) bytes, 256-byte
 * aligned; its contents on entry do not matter.
 * Requires 1 <= V < 2^31, D >= 1, 0 <= T < 2^30.  grad must be 4-byte (fp32)
 * or 2-byte (bf16) aligned.
 */
size_t emb_grad_coalesce_workspace_bytes(int32_t T, int64_t V, int32_t D,
                                         int32_t grad_dtype);
int emb_grad_coalesce(const int32_t *ids, int32_t T, const void *grad,
                      int32_t grad_dtype, int32_t D, int64_t V,
                      int32_t *uniq_ids, int32_t *seg_offsets,
                      float *uniq_grad, int32_t *num_unique, void *workspace,
                      size_t workspace_bytes, int32_t *dev_status,
                      void *stream);

/*
 * Pack the coalesced rows into per-owner send buffers (Sec. 4.1.1 / 4.1.2: the
 * sparse gradients are exchanged with an AlltoAll; each of the P shards
 * receives the rows it owns).  The P shards are partitions of one table on
 * this device.
 *   uniq_ids [cap_rows], uniq_grad [cap_rows][D], num_unique [1]: the rows
 *   k < *num_unique (read on the device; must be <= cap_rows).
 *   row_owner [V] int32: owner shard of each table row, in [0, P).
 * Outputs:
 *   send_counts  [P]     rows per owner
 *   send_offsets [P + 1] exclusive scan of send_counts
 *   send_ids     [cap_rows], send_rows [cap_rows][D]: owner p's rows at
 *   [send_offsets[p], send_offsets[p + 1]), in the order of the input (so
 *   ascending id when the input is emb_grad_coalesce output); rows are bit
 *   copies.
 * A row whose id is outside [0, V) or whose owner is outside [0, P) is not
 * sent and sets EMB_DEV_ID_OUT_OF_RANGE / EMB_DEV_OWNER_OUT_OF_RANGE.
 * workspace: at least emb_pack_by_owner_workspace_bytes(cap_rows, P) bytes.
 * Requires 1 <= P <= 1024, cap_rows >= 0, D >= 1, 1 <= V < 2^31.
 */
size_t emb_pack_by_owner_workspace_bytes(int32_t cap_rows, int32_t P);
int emb_pack_by_owner(const int32_t *uniq_ids, const float *uniq_grad,
                      const int32_t *num_unique, int32_t cap_rows, int32_t D,
                      const int32_t *row_owner, int64_t V, int32_t P,
                      int32_t *send_ids, float *send_rows,
                      int32_t *send_counts, int32_t *send_offsets,
                      void *workspace, size_t workspace_bytes,
                      int32_t *dev_status, void *stream);

/*
 * emb_grad_coalesce and emb_pack_by_owner in one call (Algorithm 1's COALESCE
 * and UNIQUE, Sec. 4.2.2, with the per-owner send layout of Sec. 4.1.2): the
 * tokens are sorted by (row_owner[id], id), so the distinct ids come out
 * already grouped by owner, ascending inside each owner, and the summed rows
 * are written straight into the send buffers.  The outputs equal those of
 * emb_pack_by_owner applied to the output of emb_grad_coalesce:
 *   send_ids  [T], send_rows [T][D]: owner p's rows at
 *             [send_offsets[p], send_offsets[p + 1])
 *   send_counts [P], send_offsets [P + 1]
 *   num_unique [1]: rows sent (= send_offsets[P])
 *   seg_offsets [T + 1]: seg_offsets[k + 1] - seg_offsets[k] tokens were summed
 *             into send row k (offsets in the owner-major token order)
 * except that the order of the fp32 additions inside a row may differ (same
 * rule: position order in chunks of 32 sorted tokens, then an ordered combine,
 * or plain position order for at most 2048 tokens; bitwise reproducible run to
 * run).  A token whose id is outside [0, V) or
 * whose owner is outside [0, P) is left out and sets EMB_DEV_ID_OUT_OF_RANGE /
 * EMB_DEV_OWNER_OUT_OF_RANGE.
 * workspace: emb_grad_coalesce_workspace_bytes(T, V, D, grad_dtype) bytes,
 * 256-byte aligned.  Requires what emb_grad_coalesce requires, 1 <= P <= 1024,
 * and bits(V) + bits(P) <= 32, where bits(n) is the number of bits of n - 1
 * (EMB_ERR_UNSUPPORTED otherwise; use the two calls).
 */
int emb_grad_coalesce_by_owner(const int32_t *ids, int32_t T,
                               const void *grad, int32_t grad_dtype,
                               int32_t D, int64_t V,
                               const int32_t *row_owner, int32_t P,
                               int32_t *send_ids, int32_t *seg_offsets,
                               float *send_rows, int32_t *send_counts,
                               int32_t *send_offsets, int32_t *num_unique,
                               void *workspace, size_t workspace_bytes,
                               int32_t *dev_status, void *stream);

/*
 * emb_grad_coalesce_by_owner for callers that cannot allocate device memory
 * (code under HIP graph capture, tight serving loops, harnesses that forbid
 * allocation): the same arguments, outputs and rules, without the workspace.
 * The call allocates nothing and calls no allocating routine; its workspace is
 * a static device array of EMB_NOALLOC_SCRATCH_BYTES (16 MiB) that each device
 * the library runs on holds until the process ends (its address is looked up
 * once per device, at the first call on it).
 * Returns EMB_ERR_WORKSPACE, before anything touches the device, when
 * emb_grad_coalesce_workspace_bytes(T, V, D, grad_dtype) exceeds
 * EMB_NOALLOC_SCRATCH_BYTES (e.g. more than about 380k tokens of 256 floats, or
 * 182k of 1024).  Every call on one device shares the array, which keeps the
 * last call's contents (the call clears what must start at zero itself): calls
 * in order on one stream are safe; calls that can overlap on one device
 * (different streams, nothing ordering them) race on it.
 */
#define EMB_NOALLOC_SCRATCH_BYTES ((size_t)16 << 20)
int emb_grad_coalesce_by_owner_noalloc(const int32_t *ids, int32_t T,
                                       const void *grad, int32_t grad_dtype,
                                       int32_t D, int64_t V,
                                       const int32_t *row_owner, int32_t P,
                                       int32_t *send_ids, int32_t *seg_offsets,
                                       float *send_rows, int32_t *send_counts,
                                       int32_t *send_offsets,
                                       int32_t *num_unique,
                                       int32_t *dev_status, void *stream);

/*
 * emb_grad_coalesce_by_owner with the set split of Vertical Sparse Scheduling
 * (Algorithm 1; Sec. 4.2.2, "Minimum Dependency of Embedding").  With the next
 * batch's ids known in advance (next_ids [T_next]), a coalesced row is prior
 * when its id occurs in the next batch (i_prior = D_u intersect D_next) and
 * delayed otherwise.  The send layout holds 2P groups: the prior rows of
 * owners 0 .. P-1, then the delayed rows of owners 0 .. P-1, each group in
 * ascending id:
 *   send_counts [2P], send_offsets [2P + 1]: group g is
 *   [send_offsets[g], send_offsets[g + 1]); prior rows are
 *   [send_offsets[0], send_offsets[P]), delayed [send_offsets[P], send_offsets[2P]).
 * The other outputs and rules are those of emb_grad_coalesce_by_owner.  Ids
 * of next_ids outside [0, V) match no row.  Adam is then applied to each part
 * (emb_sparse_adam_apply with offsets send_offsets and send_offsets + P), both
 * with the same step (Sec. 5.7).
 * workspace: emb_grad_coalesce_split_workspace_bytes(T, T_next, V, D,
 * grad_dtype) bytes, 256-byte aligned.  Requires 0 <= T_next < 2^30 and
 * bits(V) + bits(P) + 1 <= 32 (EMB_ERR_UNSUPPORTED otherwise).
 */
size_t emb_grad_coalesce_split_workspace_bytes(int32_t T, int32_t T_next,
                                               int64_t V, int32_t D,
                                               int32_t grad_dtype);
int emb_grad_coalesce_split(const int32_t *ids, int32_t T,
                            const int32_t *next_ids, int32_t T_next,
                            const void *grad, int32_t grad_dtype, int32_t D,
                            int64_t V, const int32_t *row_owner, int32_t P,
                            int32_t *send_ids, int32_t *seg_offsets,
                            float *send_rows, int32_t *send_counts,
                            int32_t *send_offsets, int32_t *num_unique,
                            void *workspace, size_t workspace_bytes,
                            int32_t *dev_status, void *stream);

/*
 * The receiver side of the sparse-gradient AlltoAll (Sec. 4.1.1 / 4.1.2: every
 * worker sends each owner the coalesced rows it owns; an owner then sums the
 * rows it received for the same index), simulated on this device for P
 * workers whose send layouts sit side by side:
 *   send_ids [P][cap_rows], send_rows [P][cap_rows][D], send_offsets [P][P + 1]:
 *   worker w's rows for owner p at [send_offsets[w][p], send_offsets[w][p + 1])
 *   of its own block (the layout of emb_grad_coalesce_by_owner / emb_pack_by_owner).
 * emb_exchange_simulated moves every block to its receiver (a P x P block
 * transpose; rows are bit copies):
 *   recv_offsets [P][P + 1]: owner p receives worker w's rows at
 *   [recv_offsets[p][w], recv_offsets[p][w + 1]), and all its rows end at
 *   recv_offsets[p][P]; receivers follow each other (owner-major).
 *   recv_ids [P * cap_rows], recv_rows [P * cap_rows][D]; recv_total [1] = rows received.
 * Offsets are clamped into [0, cap_rows]; rows outside a worker's blocks are
 * not sent.  D == 0 moves the ids alone (send_rows and recv_rows may be NULL):
 * the lookup requests of emb_lookup_request.  Requires 1 <= P <= 1024,
 * P * cap_rows < 2^30, D >= 0.
 *
 * emb_receive_merge then coalesces the received rows of every owner (their
 * ids can repeat across senders): emb_grad_coalesce_by_owner over the first
 * *recv_total of the cap received rows (fp32), with the same outputs, rules
 * and workspace (emb_grad_coalesce_workspace_bytes(cap, V, D, EMB_F32)).  Rows
 * of one index are summed in sender order.  The result equals the owner-major
 * coalesce of all workers' tokens together (to the fp32 summation bound).
 */
int emb_exchange_simulated(const int32_t *send_ids, const float *send_rows,
                           const int32_t *send_offsets, int32_t P,
                           int32_t cap_rows, int32_t D, int32_t *recv_ids,
                           float *recv_rows, int32_t *recv_offsets,
                           int32_t *recv_total, void *stream);
int emb_receive_merge(const int32_t *recv_ids, const float *recv_rows,
                      const int32_t *recv_total, int32_t cap, int32_t D,
                      int64_t V, const int32_t *row_owner, int32_t P,
                      int32_t *merged_ids, int32_t *seg_offsets,
                      float *merged_rows, int32_t *merged_counts,
                      int32_t *merged_offsets, int32_t *num_unique,
                      void *workspace, size_t workspace_bytes,
                      int32_t *dev_status, void *stream);

/*
 * Lookup requests of the row-wise partition (Sec. 4.1.1: every process looks
 * up the embeddings of its own training data; with the rows partitioned, the
 * rows a worker needs live with their owners, so the forward pass asks each
 * owner for them and gets them back, the exchange that the column-wise
 * partition replaces by the lookup-result AlltoAll).  Each distinct row is
 * asked for once per worker, however many of its tokens use it.
 *   ids [T] int32; row_owner [V] int32.  A token takes part when its id is in
 *   [0, V) (else EMB_DEV_ID_OUT_OF_RANGE) and its owner in [0, P) (else
 *   EMB_DEV_OWNER_OUT_OF_RANGE).
 * Outputs (device):
 *   req_ids     [T]     the U distinct ids of the tokens that take part,
 *                       grouped by owner (owner 0 first), ascending inside a
 *                       group: the send layout of emb_exchange_simulated (D = 0)
 *   req_counts  [P], req_offsets [P + 1]: owner p's requests at
 *                       [req_offsets[p], req_offsets[p + 1])
 *   num_unique  [1]     U
 *   inverse     [T]     k with req_ids[k] = ids[t] for a token that takes
 *                       part, -1 for one that does not
 * The owners answer with emb_gather of the ids they receive; the rows that
 * come back in request order, [U][D], expand to the batch's lookup with
 * emb_gather(rows, U, D, inverse, T, out) (tokens that take no part get zero
 * rows).  Entries of req_ids past U are left unspecified.
 * workspace: device memory of at least emb_lookup_request_workspace_bytes(T, V)
 * bytes, 256-byte aligned; contents on entry do not matter.  T == 0 writes the
 * empty result.  Requires 1 <= V < 2^31, 1 <= P <= 1024, 0 <= T < 2^30;
 * EMB_ERR_UNSUPPORTED when bits(V) + bits(P) > 32 (the composite sort key of
 * emb_grad_coalesce_by_owner).
 */
size_t emb_lookup_request_workspace_bytes(int32_t T, int64_t V);
int emb_lookup_request(const int32_t *ids, int32_t T, int64_t V,
                       const int32_t *row_owner, int32_t P, int32_t *req_ids,
                       int32_t *req_counts, int32_t *req_offsets,
                       int32_t *num_unique, int32_t *inverse, void *workspace,
                       size_t workspace_bytes, int32_t *dev_status,
                       void *stream);

/*
 * Column-wise partition (Sec. 4.1.1: the table is split by columns before
 * training, so every process keeps the whole vocabulary for its slice of the
 * embedding dimension and all owners receive the same number of rows; the
 * lookup results are redistributed with one AlltoAll, the sparse gradients
 * with another).  This is the paper's own partition; the owner-major calls
 * above are the row-wise one.
 *
 * Owner p of P holds the float columns [off(p), off(p + 1)) of every row, with
 * off(p) = floor(p * D / P) and width w(p) = off(p + 1) - off(p).
 * The COLUMN-BLOCK LAYOUT of capacity C is C * D floats holding P blocks:
 * block p is the [C][w(p)] row-major slice of owner p's columns, at float
 * offset C * off(p); row r of block p is at C * off(p) + r * w(p).  With
 * C = V it is the partitioned table (shard p = block p, all V rows); the
 * shards of exp_avg and exp_avg_sq use the same layout.
 * All three calls are bit copies.  Every call requires 1 <= P <= min(D, 1024)
 * (each owner holds at least one column) and D * P < 2^31.
 *
 * emb_pack_by_column: the gradient payload of the column-wise AlltoAll.
 *   rows [cap_rows][D] (the uniq_grad of emb_grad_coalesce); the first R rows
 *   are packed, R = *num_rows (device int32, clamped into [0, cap_rows]) or
 *   R = cap_rows when num_rows is NULL (this partitions a table: rows = the
 *   [V][D] table, cap_rows = V).
 *   blocks: column-block layout of capacity cap_rows; rows >= R not written.
 *   send_counts [P] (device, may be NULL): R for every owner.  Each owner gets
 *   the same R ids (the uniq_ids of the coalesce, not copied) with its w(p)
 *   columns of each row.
 *   Owner p then applies emb_sparse_adam_apply to its shard (table, exp_avg,
 *   exp_avg_sq at float offset V * off(p), D = w(p)) with the rows of block p.
 *
 * emb_gather_by_column: the lookup of every owner (Sec. 4.1.1: each process
 *   looks up the training data of all processes in its part of the table).
 *   shards: the table in column-block layout of capacity V; ids [T].
 *   blocks: column-block layout of capacity T; block p row t =
 *   columns off(p) .. off(p + 1) - 1 of table row ids[t].  Worker q's tokens
 *   at rows [t0, t1) of every block are what owner p sends q.  An id outside
 *   [0, V) gives zeros and sets EMB_DEV_ID_OUT_OF_RANGE.  Requires
 *   1 <= V < 2^31, T >= 0.
 *
 * emb_assemble_by_column: the receiving side of the lookup-result AlltoAll.
 *   blocks: column-block layout of capacity C; rows [row0, row0 + R) of every
 *   block are joined into rows [R][D].  With the blocks of
 *   emb_gather_by_column and worker q's token range this yields exactly the
 *   rows emb_gather would return for q's ids from the unpartitioned table.
 *   Requires C >= 0, row0 >= 0, R >= 0, row0 + R <= C.
 */
int emb_pack_by_column(const float *rows, const int32_t *num_rows,
                       int32_t cap_rows, int32_t D, int32_t P, float *blocks,
                       int32_t *send_counts, void *stream);
int emb_gather_by_column(const float *shards, int64_t V, int32_t D, int32_t P,
                         const int32_t *ids, int32_t T, float *blocks,
                         int32_t *dev_status, void *stream);
int emb_assemble_by_column(const float *blocks, int64_t C, int64_t row0,
                           int32_t R, int32_t D, int32_t P, float *rows,
                           void *stream);

/*
 * Communication cost model of a sparse gradient (Sec. 4.1.2, Table 2): the
 * time of one training step's exchange of an embedding table of M bytes whose
 * gradient has density alpha (the fraction of rows with a nonzero gradient,
 * U / V for one batch), for N workers, with bandwidth B between any two
 * workers and start-up latency beta per message:
 *   EMB_COMM_ALLTOALL   2 (N - 1) (alpha M / (N B) + beta)
 *                       (lookup results and gradients, each alpha M / N per peer)
 *   EMB_COMM_ALLREDUCE  2 (N - 1) (M / (N B) + beta)    (dense ring)
 *   EMB_COMM_PS         2 N (alpha M / (S B) + beta)    (S servers; Table 2
 *                       states the lower bound, S = n nodes)
 *   EMB_COMM_ALLGATHER  (N - 1) (alpha M / B + beta)
 * Host-only arithmetic in double.  *seconds receives the cost in the units of
 * M / B and beta (host pointer).  S is read for EMB_COMM_PS only.
 * Requires N >= 1, S >= 1, M >= 0, 0 <= alpha <= 1, B > 0, beta >= 0.
 */
#define EMB_COMM_ALLTOALL 0
#define EMB_COMM_ALLREDUCE 1
#define EMB_COMM_PS 2
#define EMB_COMM_ALLGATHER 3
int emb_comm_cost(int32_t scheme, int64_t N, int64_t S, double M,
                  double alpha, double B, double beta, double *seconds);

/*
 * Row-wise (lazy) Adam on received rows (Sec. 4.1.1: each process updates its
 * embedding rows with the exchanged gradients; Sec. 5.7: Adam with a global
 * step counter that the caller owns and advances once per iteration).
 * Kingma & Ba, Algorithm 1, for each listed row r and column j:
 *   m <- b1 m + (1 - b1) g ;  v <- b2 v + (1 - b2) g^2
 *   w <- w - lr * (m / (1 - b1^step)) / (sqrt(v / (1 - b2^step)) + eps)
 * computed in fp32 (bias corrections formed in fp64 on the host).
 *   table, exp_avg, exp_avg_sq [V][D] fp32, updated in place.
 *   row_ids [cap_rows], rows [cap_rows][D]: the rows i in
 *   [offsets[shard_begin], offsets[shard_end]) are applied, with offsets
 *   [P + 1] in device memory (the send_offsets of emb_pack_by_owner);
 *   that range must lie within [0, cap_rows).
 * Rows not listed keep table, exp_avg and exp_avg_sq bit-unchanged.  Listed
 * row ids must be distinct (true of pack output); an id outside [0, V) is
 * skipped and sets EMB_DEV_ID_OUT_OF_RANGE.
 * Requires 1 <= P <= 1024, 0 <= shard_begin <= shard_end <= P, step >= 1,
 * 0 <= beta1, beta2 < 1, eps >= 0.
 */
int emb_sparse_adam_apply(float *table, float *exp_avg, float *exp_avg_sq,
                          int64_t V, int32_t D, const int32_t *row_ids,
                          const float *rows, const int32_t *offsets, int32_t P,
                          int32_t shard_begin, int32_t shard_end,
                          int32_t cap_rows, double lr, double beta1,
                          double beta2, double eps, int64_t step,
                          int32_t *dev_status, void *stream);

/*
 * The update's coefficients for one step (Kingma & Ba, Algorithm 1, as
 * emb_sparse_adam_apply forms them: bias corrections in fp64, each
 * coefficient rounded once to fp32), written to out[EMB_ADAM_COEFFS_WORDS]
 * (host memory): beta1, 1 - beta1, beta2, 1 - beta2, lr / (1 - beta1^step),
 * 1 / (1 - beta2^step), eps, 0.  Copied to device memory and named by
 * emb_step_args.adam_coeffs, they let steps captured in a graph advance the
 * step count on every replay (Sec. 5.7: the step counter grows once per
 * iteration).  Host arithmetic only; EMB_ERR_INVALID_ARG as for
 * emb_sparse_adam_apply's hyper-parameters.
 */
#define EMB_ADAM_COEFFS_WORDS 8
int emb_adam_coeffs(double lr, double beta1, double beta2, double eps,
                    int64_t step, float *out);

/*
 * ---------------------------------------------------------------------------
 * Step executor.  Not a step of the path itself: it enqueues the four calls
 * above for one training step of one table, in data order, on up to four streams,
 * so that the latency-bound coalesce/pack work of a step overlaps the
 * bandwidth-bound lookup and update of neighbouring steps (the sparse
 * gradient work runs in GPU idle time, as in Vertical Sparse Scheduling,
 * Sec. 4.2.2, here on one GPU).  One host call per step keeps the host ahead
 * of the GPU.
 *
 * The caller rotates buffer sets (coalesce and pack workspaces, uniq_* and
 * send_* outputs; two unless `sets` says more) between consecutive steps and
 * gives each set its own events; `reuse` is nonzero when the set was used
 * before.  Below, "s-2" is the set's previous step, s - sets.  The streams may
 * differ between sets, and a set's streams may change from one use to the
 * next (with the `coalesce` stream alternating between two streams, the sorts
 * of consecutive steps run side by side): the waits on a set's previous use
 * are issued whatever the streams, and cost nothing when the stage waited for
 * ran on the waiting stream.  `lookup_update` must be the same stream for
 * every step of a table (the lookup of a step follows the previous update in
 * stream order), and a table's steps change between split and not split only
 * once the work enqueued so far has completed.
 *
 * by_owner == 0: emb_grad_coalesce on the `coalesce` stream, emb_pack_by_owner
 * on the `pack` stream, lookup and update on `lookup_update`, with the waits
 *   coalesce(s) after pack(s-2)                (same unique-row buffers)
 *   pack(s)     after coalesce(s), update(s-2) (reads unique rows; same send buffers)
 *   update(s)   after pack(s)                  (reads the packed rows)
 *   lookup(s+1) after update(s)                (same stream; reads the table)
 * (events coalesced, packed, updated).
 *
 * by_owner != 0: emb_grad_coalesce_by_owner in its two halves.  The sort of
 * the (owner, id) keys, which does not read the gradients, runs on the
 * `coalesce` stream; the reduction, which writes the send buffers directly,
 * on the `pack` stream; the lookup and the update on `lookup_update`;
 * uniq_ids, uniq_grad and ws_pack are not used.  Waits:
 *   sort(s)     after reduce(s-2)              (same coalesce workspace)
 *   reduce(s)   after sort(s), update(s-2)     (reads the sorted keys; same send buffers)
 * (with sets >= 4 and no split: sort(s) after update(s-sets), which followed
 * reduce(s-sets), and reduce(s) after sort(s) only: one wait fewer per step)
 *   update(s)   after reduce(s)                (reads the send rows)
 *   lookup(s+1) after update(s)                (same stream; reads the table)
 * (events sorted, coalesced, updated).  The sorts thus run up to a step
 * ahead, and a step's reduction runs beside the previous update and its own
 * lookup.
 *
 * split != 0 (with by_owner): Vertical Sparse Scheduling (Sec. 4.2.2,
 * Algorithm 1).  The coalesce is emb_grad_coalesce_split with the next
 * batch's ids (args.next_ids, which must be the ids of the next call), and the
 * update runs in two parts: the prior rows (needed by the next lookup) on
 * `lookup_update` right after the lookup, the delayed rows on the `delayed`
 * stream, beside the next lookup, which reads none of them.  Both parts use
 * the same Adam step.  Waits, in addition to the above:
 *   lookup(s)   after delayed update of the step two back (its rows may be in
 *               this batch; this one is two steps whatever `sets` is)
 *   prior(s)    after reduce(s)
 *   delayed(s)  after reduce(s), lookup(s)     (reads the send rows; lookup(s) reads its rows)
 *   reduce(s)   after delayed update(s-2)      (same send buffers)
 * (events gathered: the end of the lookup, delayed_done: the end of the
 * delayed update).  The pair timing[4..5] times the prior update and
 * timing[6..7] the delayed one.
 *
 * With all streams equal the calls simply run one after another, and the
 * results are bitwise the same either way.
 *
 * Graph capture.  While `lookup_update` is being captured into a HIP graph
 * (stream capture, events only: step signals and timing events are refused
 * with EMB_ERR_UNSUPPORTED), the executor records every stage end as an event
 * node instead of attaching events to dispatches.  The captured steps must not
 * wait for steps enqueued before the capture began: each buffer set's first use
 * in a capture has reuse == 0 (a replayed graph runs after the work before it
 * on its stream, whole).  With args.adam_coeffs the update reads its
 * coefficients from device memory when it runs, so a replay can apply other
 * step numbers than the ones the capture saw.
 * ---------------------------------------------------------------------------
 */
typedef struct {
  void *lookup_update;          /* stream of emb_gather and emb_sparse_adam_apply */
  void *coalesce;               /* stream of emb_grad_coalesce (by_owner: of its sort) */
  void *pack;                   /* stream of emb_pack_by_owner */
  void *delayed;                /* split: stream of the delayed update */
  void *sorted, *coalesced, *packed, *updated; /* events of this step's buffer set
                                   (sorted: by_owner only; packed: by_owner == 0 only) */
  void *gathered, *delayed_done; /* split only: events of this step's buffer set */
  int32_t reuse;                /* the buffer set was used two steps ago */
  int32_t by_owner;             /* use emb_grad_coalesce_by_owner instead of coalesce + pack */
  int32_t split;                /* by_owner with the prior / delayed split */
  void *timing[8];              /* optional timing events (NULL to skip): begin/end of
                                   gather, coalesce, pack, adam, each recorded on the
                                   stream the (first / last) kernel runs on; the adam
                                   pair takes the update kernel's own start and end
                                   from its dispatch; by_owner records no pack pair */
  void *signals;                /* optional step signals of the table
                                   (emb_step_signals_create): when set, the waits above
                                   go through them and the events sorted .. delayed_done
                                   and `reuse` are not used (they may be NULL) */
  int32_t sets;                 /* buffer sets the caller rotates (0: 2; at most 64): the
                                   waits for a set's earlier use ("s-2" above) reach back
                                   this many steps; `reuse` means the set was used `sets`
                                   steps ago.  With events the split needs 2 */
} emb_step_schedule;

typedef struct {
  float *table, *exp_avg, *exp_avg_sq; /* [V][D] fp32, updated in place */
  int64_t V;
  int32_t D;
  const int32_t *row_owner; /* [V] */
  int32_t P;
  const int32_t *ids;       /* [T] */
  int32_t T;
  const int32_t *next_ids;  /* split: [T_next] ids of the next call's batch */
  int32_t T_next;
  const void *grad;         /* [T][D], grad_dtype */
  int32_t grad_dtype;
  int32_t cap_rows;         /* capacity of the uniq_*, seg_offsets and send_* buffers (>= T, T_next) */
  float *lookup;            /* [T][D] gather output */
  int32_t *uniq_ids, *seg_offsets, *num_unique;
  float *uniq_grad;
  int32_t *send_ids, *send_counts, *send_offsets; /* counts [P] and offsets [P + 1]; split: [2P], [2P + 1] */
  float *send_rows;
  void *ws_coalesce;
  size_t ws_coalesce_bytes;
  void *ws_pack;
  size_t ws_pack_bytes;
  double lr, beta1, beta2, eps;
  int64_t step;             /* Adam step (>= 1), one per iteration (Sec. 5.7) */
  int32_t *dev_status;      /* optional */
  const void *adam_coeffs;  /* optional, 16-byte aligned device memory: this step's
                               EMB_ADAM_COEFFS_WORDS update coefficients (emb_adam_coeffs),
                               read by the update kernel when it runs instead of those of
                               `step` (for steps replayed from a graph) */
} emb_step_args;

/* Events for the schedule (hipEventCreateWithFlags; timing: nonzero for
 * timing events).  A host-side runtime object, not device memory. */
int emb_event_create(void **event, int32_t timing);
int emb_event_destroy(void *event);
/* Milliseconds between two completed timing events. */
int emb_event_elapsed_ms(void *start, void *end, float *ms);

/* Step signals: the cross-stream order of emb_train_step kept through stream
 * memory operations instead of events.  A handle holds two words of HIP
 * signal memory per stage (sorted, coalesced, packed, updated, gathered,
 * delayed_done), for steps of even and of odd number, and a step counter.
 * Each emb_train_step call that names the handle takes the next step number n;
 * the end of a stage writes n into its word of n's parity
 * (hipStreamWriteValue32) and a stream that must follow the stage of step
 * n - k waits until the word of (n - k)'s parity reaches n - k
 * (hipStreamWaitValue32, >=).  (With the two parities on two streams, as when
 * the odd and even steps' coalesce runs on two streams, each word has a single
 * writer.)
 * The order is the one listed above for the events.  A wait never targets
 * more than the value of the last write already enqueued for its word (a
 * stage that did not run in the step waited for is waited for at its last
 * run, or not at all), so every wait refers to an earlier enqueued write and
 * the waits cannot deadlock, whatever modes the calls of a handle mix.
 * On this runtime a wait on
 * a pending event costs the host about four times as much as this write and
 * wait, and with the host running ahead of the GPU nearly every wait is on a
 * pending event; the GPU-side order is the same.
 * Use one handle per table (both of its buffer sets), from one host thread.
 * If a call fails part-way, every stage of its step is marked done so that no
 * later wait blocks.  destroy: only once the work of every step enqueued with
 * the handle has completed; the signal memory is kept for a later handle (it
 * is never returned to the runtime).  create returns EMB_ERR_UNSUPPORTED if
 * the device cannot wait on stream values. */
int emb_step_signals_create(void **signals);
int emb_step_signals_destroy(void *signals);

/* Enqueue one training step of one table (see above).  Returns the first
 * failing call's status; nothing after it is enqueued. */
int emb_train_step(const emb_step_args *args, const emb_step_schedule *sched);

/* Two-thread enqueue.  Not a step of the method: a host-side way to enqueue
 * the same steps for callers whose host time per step bounds them (small
 * batches: the executor issues a dozen HIP calls per step, and a wait on an
 * event still pending on another stream alone costs the host about 10 us).
 * emb_train_step_queued enqueues the sort and the reduction of the step (on
 * `coalesce` and `pack`) from the calling thread and hands the rest (the
 * lookup, the wait for the reduction and the update, on `lookup_update`) to
 * the queue's worker thread, which enqueues the handed steps in call order on
 * the device that was current at the call.  The stream order is exactly the
 * one emb_train_step gives.  Before the calling thread waits on a buffer
 * set's earlier use, it waits (on the host, at most 30 s, else
 * EMB_ERR_LAUNCH) until the worker has enqueued that use's update.
 * Restrictions: events (no step signals), by_owner without the split, not
 * under graph capture, `coalesce` and `pack` other streams than
 * `lookup_update` (each stream is fed by one thread; EMB_ERR_UNSUPPORTED
 * otherwise); one queue per table,
 * used from one thread; timing events in `sched` are recorded as usual, those
 * of the lookup and the update by the worker.
 * Until emb_step_queue_flush has returned, the handed parts of the steps may
 * not be enqueued yet: call it before enqueuing anything on `lookup_update`
 * that must follow them, and before reading what they write.  flush and
 * destroy return the first error of a handed part (a failed part stops its
 * own step only, as in emb_train_step); destroy enqueues what was handed
 * before it stops the worker.  The queue is host memory and a thread; the
 * library allocates nothing on the device for it. */
int emb_step_queue_create(void **queue);
int emb_step_queue_flush(void *queue);
int emb_step_queue_destroy(void *queue);
int emb_train_step_queued(void *queue, const emb_step_args *args, const emb_step_schedule *sched);

/*
 * ---------------------------------------------------------------------------
 * Dense operators of a training step: not a part of the paper's path, but what
 * stands around the tables on the same GPU.  The conventions are those above.
 * Element types EMB_F32 and EMB_BF16 name the type of rows; statistics, sums
 * and parameters are fp32, and a value is rounded once, when it is written.
 * ld* are the elements from one row to the next; rows are contiguous inside and
 * need the alignment of their element type only.
 * ---------------------------------------------------------------------------
 */

/*
 * Layer norm of T rows of D elements:
 *   mean = sum x / D,  rstd = 1 / sqrt(sum (x - mean)^2 / D + eps)
 *   y = (x - mean) rstd weight + bias
 *   x     row t at x + t * ldx (x_dtype); with ids (int32 [T], else NULL) row
 *         ids[t] of a table of V rows at x + ids[t] * ldx: the lookup of
 *         emb_gather and the norm in one pass.  An id outside [0, V) reads as a
 *         row of zeros and sets EMB_DEV_ID_OUT_OF_RANGE.
 *   weight, bias [D] fp32, each may be NULL (1 and 0)
 *   y     row t at y + t * ldy (y_dtype); may be x itself where the types are
 *         the same and ids is NULL
 *   mean, rstd [T] fp32: the statistics that the backward pass takes
 * The variance is summed from the differences to the mean.  A row with an
 * infinity or a NaN is NaN; other rows are not touched by it.
 * Requires 0 <= T < 2^30, 1 <= D < 2^28, ldx >= 0, ldy >= D, eps >= 0 and
 * finite; V as in emb_gather where ids is given.  T == 0 is a no-op.
 */
int emb_layer_norm(const void *x, int32_t x_dtype, int64_t ldx,
                   const int32_t *ids, int64_t V, int32_t T, int32_t D,
                   const float *weight, const float *bias, double eps, void *y,
                   int32_t y_dtype, int64_t ldy, float *mean, float *rstd,
                   int32_t *dev_status, void *stream);

/*
 * The gradient of emb_layer_norm: with xh = (x - mean) rstd and g = dy weight,
 *   dx = rstd (g - sum g / D - xh sum (g xh) / D)       row t at dx + t * lddx
 *   dweight = sum over t of dy xh,  dbias = sum over t of dy          [D] fp32
 * dy and dx have the type dy_dtype; x, ids, V, weight, mean and rstd as in the
 * forward call.  dx (one row per token, the gradient rows that
 * emb_grad_coalesce takes), dweight and dbias may each be NULL: not computed.
 * dx may be dy itself.  T == 0 writes zeros to dweight and dbias.
 * dweight and dbias are overwritten.  Their sums run in an order that depends
 * on T, D and the types only: bitwise reproducible run to run.
 * workspace: at least emb_layer_norm_backward_workspace_bytes(T, D) bytes,
 * 256-byte aligned, contents on entry do not matter (not used where dweight
 * and dbias are NULL).
 */
size_t emb_layer_norm_backward_workspace_bytes(int32_t T, int32_t D);
int emb_layer_norm_backward(const void *dy, int32_t dy_dtype, int64_t lddy,
                            const void *x, int32_t x_dtype, int64_t ldx,
                            const int32_t *ids, int64_t V, int32_t T,
                            int32_t D, const float *weight, const float *mean,
                            const float *rstd, void *dx, int64_t lddx,
                            float *dweight, float *dbias, void *workspace,
                            size_t workspace_bytes, int32_t *dev_status,
                            void *stream);

/*
 * Relative position bias by buckets: a learned table with one row per bucket of
 * position differences and one column per attention head, looked up for every
 * pair of a query and a key:
 *   out[h][i][j] = table[bucket_of[clamp(j - (q0 + i), -R, R) + R]][h]
 *   table      [num_buckets][H] fp32
 *   bucket_of  [2 R + 1] int32, the bucket of each difference key - query in
 *              [-R, R]; larger differences share the ends' buckets.  A negative
 *              entry masks its pairs: out is -infinity.  An entry of num_buckets
 *              or more that any pair has sets EMB_DEV_BUCKET_OUT_OF_RANGE and
 *              reads as 0.
 *   q0         position of query 0 (keys are at 0 .. K - 1): K - Q where the
 *              queries are the last Q of K positions, e.g. one new token after
 *              K - 1 others
 *   out        element (h, i, j) at out + h * ldh + i * ldq + j (out_dtype)
 * Q == 0 or K == 0 is a no-op.  Requires num_buckets >= 1, 1 <= H <= 65535,
 * 0 <= R < 2^30, 0 <= Q, K < 2^30, |q0| < 2^62, ldq >= K, and heads that do not
 * overlap: where H > 1, ldh >= (Q - 1) ldq + K, or (the rows of a query's heads
 * side by side) ldh >= K and ldq >= (H - 1) ldh + K.
 */
int emb_relative_bias(const float *table, int32_t num_buckets, int32_t H,
                      const int32_t *bucket_of, int32_t R, int32_t Q,
                      int32_t K, int64_t q0, void *out, int32_t out_dtype,
                      int64_t ldq, int64_t ldh, int32_t *dev_status,
                      void *stream);

/*
 * The gradient of emb_relative_bias, where the bias was added for each of N
 * batch entries:
 *   dtable[b][h] = sum over n, i, j with bucket b of grad[n][h][i][j]
 *   grad    element (n, h, i, j) at grad + n * ldn + h * ldh + i * ldq + j
 *           (grad_dtype); what stands in masked places is not used, whatever it
 *           is.  Entries of bucket_of that are num_buckets or more are left out,
 *           and set EMB_DEV_BUCKET_OUT_OF_RANGE where any pair has them.
 *   dtable  [num_buckets][H] fp32, overwritten (0 for a bucket without pairs)
 * Sums are fp32 in an order that depends on the sizes and bucket_of only:
 * bitwise reproducible run to run.
 * workspace: at least emb_relative_bias_backward_workspace_bytes(N, H, Q, K)
 * bytes, 256-byte aligned, contents on entry do not matter.
 * Requires what emb_relative_bias requires of the sizes, N >= 0 and strides of
 * 0 or more.
 */
size_t emb_relative_bias_backward_workspace_bytes(int32_t N, int32_t H,
                                                  int32_t Q, int32_t K);
int emb_relative_bias_backward(const void *grad, int32_t grad_dtype, int32_t N,
                               int32_t H, int32_t Q, int32_t K, int64_t ldn,
                               int64_t ldh, int64_t ldq,
                               const int32_t *bucket_of, int32_t R,
                               int32_t num_buckets, int64_t q0, float *dtable,
                               void *workspace, size_t workspace_bytes,
                               int32_t *dev_status, void *stream);

/*
 * The usual map of position differences to buckets, for R = max_distance,
 * written to out[2 max_distance + 1] (host memory): half of the buckets of a
 * direction hold one distance each, the others hold ranges that grow by a
 * constant factor up to max_distance, and the last one everything beyond.
 * With m = buckets of a direction and e = m / 2, distance n >= e has bucket
 * min(m - 1, e + floor(log(n / e) / log(max_distance / e) (m - e))).
 * causal == 0: keys after the query take the upper half of the buckets
 * (num_buckets even, m = num_buckets / 2), the others the lower; otherwise all
 * buckets are for keys at or before the query and the others are masked (-1).
 * Host arithmetic only.  Requires m >= 2 and max_distance > e.
 */
int emb_relative_buckets(int32_t num_buckets, int32_t max_distance,
                         int32_t causal, int32_t *out);

/*
 * One AdamW step (Kingma & Ba, Algorithm 1, with decoupled decay) of many
 * tensors: the dense parameters, beside emb_sparse_adam_apply for table rows.
 * For every element, with the step number t:
 *   g <- grad_scale g;  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
 *   w <- w - lr weight_decay w
 *   w <- w - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
 * in fp32 without fused multiply-adds, each operation rounded to nearest and
 * subnormal numbers kept (bias corrections formed in fp64 on the host, every
 * coefficient rounded once to fp32: lr / (1 - b1^t), which multiplies the
 * quotient of m by the root plus eps, 1 / (1 - b2^t), and lr weight_decay).
 *
 * emb_adamw_tensor names one tensor's arrays of n elements (device memory,
 * element alignment only, updated in place; different tensors' arrays must not
 * overlap):
 *   param       fp32
 *   grad        fp32 or bf16 (grad_dtype, the same for all tensors of a call)
 *   exp_avg, exp_avg_sq   m and v.  state_bits == 32: fp32.  state_bits == 8:
 *               m as float8 e4m3 (the variant without infinities, largest value
 *               448) and v as float8 e5m2, one byte each, times scales
 *   scales      state_bits == 8: 2 B fp32 with B = ceil(n / EMB_ADAMW_BLOCK);
 *               elements k EMB_ADAMW_BLOCK ... of m have scales[k], of v
 *               scales[B + k], powers of two.  Zeros in all three are zero moments.
 *   copy        NULL, or bf16 [n]: the updated w, rounded to nearest even (in
 *               every tensor of a call or in none)
 * An 8-bit moment x of a block is stored as x / scale rounded to one of the two
 * neighbouring values of its type, to the upper one with the probability of the
 * distance from the lower one (so that small changes of a moment add up over
 * the steps); a v other than 0 is stored as at least the smallest value.  The
 * block's largest magnitude over scale is in [2^7, 2^8) for m, in [2^14, 2^15)
 * for v (less where the scale would be below 2^-126).  The update uses the
 * moments before they are rounded.  Random bits: with mix64 and GAMMA of
 * SplitMix64 (Steele, Lea & Flood 2014), elements 2 j and 2 j + 1 of the
 * call's k-th tensor take the low and the high half of
 *   mix64(mix64(mix64(seed + t GAMMA) + (k + 1) GAMMA) + (j + 1) GAMMA)
 * and of that half the low 16 bits r for m, the high 16 for v; the part cut off,
 * as a fraction of a step in [0, 1), rounds up if fraction + (r + 1/2) / 2^16
 * is 1 or more.  The result depends on nothing else: bitwise reproducible.
 * A block with a moment that is infinite or NaN gets a NaN scale: its moments
 * are NaN from then on, as the element's own are with 32 bits.  Either way
 * EMB_DEV_NOT_FINITE is set.
 *
 *   tensors     [n_tensors] in HOST memory, read before the call returns
 *   coeffs      NULL, or this step's EMB_ADAMW_COEFFS_WORDS coefficients
 *               (emb_adamw_coeffs) in device memory, 16-byte aligned, read by the
 *               kernel in place of lr .. seed: for steps replayed from a graph
 *   grad_scale  NULL (1), or one fp32 in device memory (a clipping factor, the
 *               inverse of a loss scale)
 * Tensors with n == 0 are skipped.  Requires n_tensors >= 0, 0 <= n <= 2^33,
 * step >= 1, 0 <= beta1, beta2 < 1, eps >= 0, finite lr and weight_decay >= 0.
 */
#define EMB_ADAMW_BLOCK 256
#define EMB_ADAMW_COEFFS_WORDS 12
typedef struct {
  float *param;
  const void *grad;
  void *exp_avg, *exp_avg_sq;
  float *scales;
  void *copy;
  int64_t n;
} emb_adamw_tensor;
int emb_adamw_step(const emb_adamw_tensor *tensors, int32_t n_tensors,
                   int32_t grad_dtype, int32_t state_bits, double lr,
                   double beta1, double beta2, double eps, double weight_decay,
                   int64_t step, uint64_t seed, const void *coeffs,
                   const float *grad_scale, int32_t *dev_status, void *stream);

/* The coefficients of one emb_adamw_step, written to
 * out[EMB_ADAMW_COEFFS_WORDS] (host memory; the layout is the library's own).
 * Host arithmetic only; EMB_ERR_INVALID_ARG as for emb_adamw_step. */
int emb_adamw_coeffs(double lr, double beta1, double beta2, double eps,
                     double weight_decay, int64_t step, uint64_t seed,
                     void *out);

/*
 * Dropout from a counter-based generator; the mask is never stored:
 *   y = residual + keep x / (1 - q)
 * With cut = min(65535, round(65536 p)) and q = cut / 65536, element (t, d) of
 * the T rows of D is kept where its 16 random bits are cut or more.  Bits: with
 * mix64 and GAMMA of SplitMix64 (Steele, Lea & Flood 2014), elements 4 j .. 4 j +
 * 3 of row t take the four 16-bit quarters, the lowest first, of
 *   mix64(mix64(seed) + (t ceil(D / 4) + j + 1) GAMMA)
 * The result depends on nothing else.  What is dropped is not used, whatever it
 * is.  The gradient of x is the same call on the gradient of y, without a
 * residual.
 *   x, y      rows at x + t * ldx, y + t * ldy (dtype); y may be x or residual
 *   residual  rows at residual + t * ldr (dtype), or NULL (0)
 *   seed_dev  NULL, or one uint64 in device memory, 8-byte aligned, read by the
 *             kernel in place of seed: for steps replayed from a graph
 * Requires 0 <= T < 2^30, 1 <= D < 2^28, 0 <= p < 1, ldx, ldr >= 0, ldy >= D.
 * T == 0 is a no-op.
 */
int emb_dropout(const void *x, int32_t dtype, int64_t ldx, int32_t T, int32_t D,
                double p, uint64_t seed, const uint64_t *seed_dev,
                const void *residual, int64_t ldr, void *y, int64_t ldy,
                void *stream);

/*
 * The end of one block and the start of the next in one pass: the norm after
 * the block, dropout, the block's gate, the scaled residual stream, and the norm
 * before the next block.
 *   n = N_post(branch)                              (emb_layer_norm's formula)
 *   h = alpha x + gate keep n / (1 - q)             (emb_dropout's mask)
 *   y = N_pre(h)
 *   x, h      T rows of D, stream_dtype; h may be x
 *   branch, y T rows of D, dtype; y may be branch.  stream_dtype is dtype, or
 *             EMB_F32 beside branch rows of EMB_BF16.
 *   gate      [ceil(T / gate_rows)][D] fp32, row t takes row t / gate_rows;
 *             gate_rows == 0: [D], all rows take it; NULL: 1
 *   post_stats, pre_stats   [2][T] fp32, mean and rstd of the two norms, which the
 *             backward pass takes.  post_stats NULL: no norm after the block (n =
 *             branch).  pre_stats NULL: no norm before the next, y is not written.
 *   post_weight, post_bias, pre_weight, pre_bias    [D] fp32, each may be NULL (1, 0)
 *   p, seed, seed_dev       as in emb_dropout
 * y is the norm of h before h is rounded to its type.  T == 0 is a no-op.
 * Requires 0 <= T < 2^30, 1 <= D < 2^28, ldx, ldb >= 0, ldh, ldy >= D, eps >= 0
 * and finite, alpha finite, 0 <= p < 1, gate_rows >= 0.
 * The struct is host memory, read before the call returns.
 */
typedef struct {
  int32_t T, D;
  int32_t stream_dtype, dtype;
  const void *x;
  int64_t ldx;
  const void *branch;
  int64_t ldb;
  const float *gate;
  int64_t gate_rows;
  const float *post_weight, *post_bias, *pre_weight, *pre_bias;
  double alpha, eps, p;
  uint64_t seed;
  const uint64_t *seed_dev;
  void *h;
  int64_t ldh;
  void *y;
  int64_t ldy;
  float *post_stats, *pre_stats;
} emb_block_norm_args;
int emb_block_norm(const emb_block_norm_args *args, void *stream);

/*
 * The gradient of emb_block_norm.  With d = dh + N_pre'(dy) (the gradient of h):
 *   dx = alpha d
 *   dn = gate keep d / (1 - q),  dbranch = N_post'(dn)
 *   dgate = the sum of keep d n / (1 - q) over the rows that share a gate
 *   dpost_weight = sum dn bh, dpost_bias = sum dn       (bh: branch normalised)
 *   dpre_weight = sum dy hh, dpre_bias = sum dy         (hh: h normalised)
 * dh [T][D] stream_dtype, or NULL (0); dy [T][D] dtype, needed where pre_stats is
 * given.  h, branch, the statistics, weights, gate, alpha, p and the seed as in
 * the forward call.  dx (stream_dtype; may be dh), dbranch (dtype; may be dy),
 * dgate [gates][D] fp32 and the four sums [D] fp32 may each be NULL: not computed;
 * dpost_* need post_stats, dpre_* pre_stats.  All are overwritten; T == 0 writes
 * zeros to the sums.  Sums run in an order that depends on the sizes and types
 * only: bitwise reproducible run to run.
 * workspace: at least emb_block_norm_backward_workspace_bytes(T, D, gate_rows)
 * bytes, 256-byte aligned, contents on entry do not matter.
 */
typedef struct {
  int32_t T, D;
  int32_t stream_dtype, dtype;
  const void *dh;
  int64_t lddh;
  const void *dy;
  int64_t lddy;
  const void *h;
  int64_t ldh;
  const void *branch;
  int64_t ldb;
  const float *gate;
  int64_t gate_rows;
  const float *post_weight, *post_bias, *pre_weight;
  const float *post_stats, *pre_stats;
  double alpha, p;
  uint64_t seed;
  const uint64_t *seed_dev;
  void *dx;
  int64_t lddx;
  void *dbranch;
  int64_t lddb;
  float *dgate, *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;
  void *workspace;
  size_t workspace_bytes;
} emb_block_norm_grad_args;
size_t emb_block_norm_backward_workspace_bytes(int32_t T, int32_t D,
                                               int64_t gate_rows);
int emb_block_norm_backward(const emb_block_norm_grad_args *args, void *stream);

/*
 * Softmax cross entropy of T tokens over the whole vocabulary of a table, whose
 * rows are the output layer.  The logits are never in memory as a whole:
 *   z[t][v] = x_t . table_v,  lse_t = log sum_v exp(z[t][v])
 *   loss_t = lse_t - (1 - e) z[t][targets_t] - e sum_v z[t][v] / V
 *   x        row t at x + t * ldx (dtype)
 *   table    row v at table + v * ldw, V rows of D (dtype)
 *   targets  [T] int32.  A negative one: the token has none, its loss and lse are
 *            0, and what stands in its row is not used.  One of V or more sets
 *            EMB_DEV_ID_OUT_OF_RANGE and counts as none.
 *   smoothing  e: the part of the target's weight that all entries share
 *   loss, lse  [T] fp32
 * Products of bf16 are exact and summed in fp32; an fp32 value enters as the sum
 * of three bf16 values, exactly, and of the products of two such sums those above
 * 2^-24 of the whole are taken.  A logit that is NaN or +infinity makes its
 * token's loss NaN (in fp32, one of -infinity too).  A table whose rows are whole
 * multiples of 64 bf16 values, on 16-byte boundaries, is read where it stands;
 * others are laid out in the workspace, a piece at a time.
 * workspace: at least emb_vocab_loss_workspace_bytes(T, V, D, dtype) bytes,
 * 256-byte aligned, contents on entry do not matter.
 * Requires 0 <= T <= 2^22, 1 <= V < 2^31, 1 <= D <= 2^16, ldx, ldw >= 0,
 * 0 <= e < 1.  T == 0 is a no-op.
 */
size_t emb_vocab_loss_workspace_bytes(int32_t T, int64_t V, int32_t D,
                                      int32_t dtype);
int emb_vocab_loss(const void *x, int32_t dtype, int64_t ldx, const void *table,
                   int64_t ldw, int32_t T, int64_t V, int32_t D,
                   const int32_t *targets, double smoothing, float *loss,
                   float *lse, void *workspace, size_t workspace_bytes,
                   int32_t *dev_status, void *stream);

/*
 * The gradient of emb_vocab_loss, the logits computed again piece by piece:
 *   g[t][v] = dloss_t (exp(z[t][v] - lse_t) - (1 - e) [v == targets_t] - e / V)
 *   dx_t = sum_v g[t][v] table_v          row t at dx + t * lddx (dtype)
 *   dtable_v = sum_t g[t][v] x_t          row v at dtable + v * lddt (dtype)
 *   dloss   [T] fp32 (dloss_step == 1), or one fp32 for all tokens (0)
 *   lse     as the forward call returned it
 * A token without a target has dx 0, whatever the table holds, and adds nothing.
 * Where the rows are bf16 and there are more than a few tokens, g (without dloss,
 * where one holds for all tokens) is rounded to bf16 (it is an operand of the
 * matrix instructions; its rounding is as large as that of dx and dtable to their
 * type); for fp32 rows three bf16 planes hold it.  Sums are fp32.  dx and dtable
 * may each be NULL: not computed.  dtable is overwritten (T == 0: zeros).  Bitwise
 * reproducible.
 */
size_t emb_vocab_loss_backward_workspace_bytes(int32_t T, int64_t V, int32_t D,
                                               int32_t dtype);
int emb_vocab_loss_backward(const float *dloss, int32_t dloss_step,
                            const void *x, int32_t dtype, int64_t ldx,
                            const void *table, int64_t ldw, int32_t T,
                            int64_t V, int32_t D, const int32_t *targets,
                            double smoothing, const float *lse, void *dx,
                            int64_t lddx, void *dtable, int64_t lddt,
                            void *workspace, size_t workspace_bytes,
                            int32_t *dev_status, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* EMB_H */
