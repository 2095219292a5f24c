/*
 * nbos -- batched replica placement for an oversubscribing notebook scheduler,
 * for NVIDIA B200 (sm_100a).  C ABI.
 *
 * The operation is the placement decision of NotebookOS (arXiv 2503.20591):
 *   Section 3.2.1  For a kernel's resource request (GPUs, VRAM GB, millicpus, memory MB) the
 *                  scheduler walks over all servers, keeps those with enough capacity, and
 *                  needs three of them, one per replica; with more than three a policy ranks
 *                  them; with fewer the caller has to scale out.
 *   Section 3.4.1  Default policy: more idle GPUs first, then the subscription ratio
 *                  SR = S / (G * R) (S subscribed GPUs, G server GPUs, R replicas per kernel);
 *                  a server whose SR would exceed the limit after placement is rejected.
 *   Section 3.2.3  A migration target must have the GPUs idle now (NBOS_REQUIRE_IDLE_GPUS).
 *
 * This library evaluates that rule for a whole batch of requests against a frozen snapshot of
 * the cluster (or against many independent snapshots at once): for every (request, host) pair
 * the feasibility test and an exact integer ranking key, then the three best distinct feasible
 * hosts per request.
 *
 * Exact definition of the result, per request (g, v, c, m) and snapshot n:
 *   host h is feasible  <=>  g,v,c,m >= 0  and  G[h] >= 1  and  g <= G[h]  and  v <= vram_gb[h]
 *                            and c <= millicpus[h] and m <= mem_mb[h]
 *                            and (S[h] + g) * limit_den[n] <= limit_num[n] * G[h] * R
 *                            and (flags & NBOS_REQUIRE_IDLE_GPUS ? g <= G[h] - C[h] : true)
 *   feasible hosts are ordered by (G-C descending, (S+g)/(G*R) ascending, h ascending)
 *   [NBOS_KEY_IDLE_FIRST, the paper's order] or by ((S+g)/(G*R) ascending, G-C descending,
 *   h ascending) [NBOS_KEY_SR_FIRST]; ratios are compared exactly.
 *   out_hosts = the first three of that order, best first, -1 where fewer exist;
 *   out_found = how many exist, capped at 3.
 *
 * Conventions
 *   - Every function returns an int status: NBOS_OK (0) or a negative NBOS_ERR_* code. Nothing
 *     throws, aborts or prints. nbos_strerror() names a code; nbos_last_error_detail() gives the
 *     calling thread's most recent failure in words.
 *   - "DEVICE" pointers are device memory of the current CUDA device; "HOST" pointers are
 *     ordinary host memory. The caller owns every buffer it passes. The library owns only the
 *     snapshot handle (host memory) and, for the *_host entry points and the host-split launch
 *     shape, stream-ordered temporary device memory that it frees itself.
 *   - `cuda_stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).
 *   - Only devices of compute capability 10.x are accepted (NBOS_ERR_UNSUPPORTED_DEVICE).
 *   - There is no CPU fallback anywhere.
 */
#ifndef NBOS_H_
#define NBOS_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define NBOS_OK 0
#define NBOS_ERR_INVALID_ARG (-1)        /* NULL / misaligned pointer, size out of range        */
#define NBOS_ERR_RANGE (-2)              /* a value in the arrays is outside what is supported  */
#define NBOS_ERR_CUDA (-3)               /* a CUDA runtime call failed                          */
#define NBOS_ERR_UNSUPPORTED_DEVICE (-4) /* current device is not compute capability 10.x       */
#define NBOS_ERR_DEVICE_TIMEOUT (-5)     /* a bounded wait inside a kernel ran out              */
#define NBOS_ERR_NO_MEMORY (-6)          /* host or device allocation failed / workspace small  */
#define NBOS_ERR_STALE_LAYOUT (-7)       /* nbos_snapshot_update: new state does not fit the key /
                                          * packing layout chosen at creation; create a new one  */

/* key_order */
#define NBOS_KEY_IDLE_FIRST 0 /* Section 3.4.1: idle GPUs, then SR, then host id (default) */
#define NBOS_KEY_SR_FIRST 1   /* SR, then idle GPUs, then host id                           */

/* flags */
#define NBOS_REQUIRE_IDLE_GPUS 1 /* Section 3.2.3: also require g <= G - C                   */
#define NBOS_FORCE_KEY64 2       /* build the 64-bit key table even if 32 bits would do      */
#define NBOS_LIMIT_CLUSTER_SR 4  /* Section 3.4.1, third factor: ignore limit_num / limit_den (they may
                                  * be NULL) and use each snapshot's own cluster-wide SR,
                                  * sum(S) / (sum(G) * R), as its limit. An empty cluster (sum S = 0)
                                  * then admits only g = 0; the paper gives no floor.          */

#define NBOS_ROOM_FOR_COMMITS 8   /* size the key's ratio field for subscribed counts growing up to each
                                  * host's cap; required by nbos_place_batch_sequential          */

#define NBOS_MAX_HOSTS (1 << 20)   /* per snapshot                          */
#define NBOS_MAX_GPUS_PER_HOST 1023
#define NBOS_MAX_REPLICAS 1024
#define NBOS_REPLICAS_PLACED 3     /* hosts returned per request (Section 3.2.1) */

typedef struct nbos_snapshot nbos_snapshot; /* opaque */

/*
 * Cluster state, structure of arrays. N snapshots of H hosts each; array element [n*H + h].
 *   gpus_total       G  (0 .. NBOS_MAX_GPUS_PER_HOST; a host with G = 0 is never feasible)
 *   gpus_subscribed  S  (>= 0)  sum of GPUs requested by all replicas scheduled on the host
 *   gpus_committed   C  (0 .. G) GPUs bound to replicas that are executing now
 *   vram_gb, millicpus, mem_mb  (>= 0) the capacity a request's ask is compared with. Pass total
 *                    capacity for the creation reading of Section 3.2.1, or what is left
 *                    unbound for the migration reading of Section 3.2.3.
 *   limit_num/limit_den  per-snapshot SR limit as a rational in the paper's units S/(G*R);
 *                    limit_num >= 0, limit_den >= 1.
 */
typedef struct nbos_snapshot_desc {
    int32_t n_snapshots; /* N >= 1                                   */
    int32_t n_hosts;     /* 1 <= H <= NBOS_MAX_HOSTS                  */
    int32_t replicas_R;  /* 1 .. NBOS_MAX_REPLICAS; the paper uses 3  */
    int32_t key_order;   /* NBOS_KEY_*                                */
    int32_t flags;       /* NBOS_REQUIRE_IDLE_GPUS | NBOS_FORCE_KEY64 | NBOS_LIMIT_CLUSTER_SR |
                          * NBOS_ROOM_FOR_COMMITS */
    int32_t reserved;    /* must be 0                                 */
    const int32_t *limit_num; /* HOST [N] in both create variants     */
    const int32_t *limit_den; /* HOST [N]                             */
    /* [N*H] each. DEVICE for nbos_snapshot_create (read by work queued on the stream: keep them
     * valid until that work has finished), HOST for nbos_snapshot_create_host (read before it
     * returns). */
    const int32_t *gpus_total, *gpus_subscribed, *gpus_committed;
    const int32_t *vram_gb, *millicpus, *mem_mb;
} nbos_snapshot_desc;

typedef struct nbos_snapshot_info {
    int32_t n_snapshots, n_hosts, hosts_padded;
    int32_t key_bits;                    /* 32 or 64: width of the ranking key in use       */
    int32_t bits_idle, bits_sr, bits_id; /* field widths inside the key                     */
    int32_t key_order, flags, replicas_R;
    int32_t packed_test; /* 0: capacities too wide for the packed test; 1: packed, one guard
                          * mask; 2: packed, one guard mask per word                        */
    int32_t static_key;  /* 1: every host has the same key slope, hosts rank the same for all g */
    int32_t presorted;   /* 1: the host table is stored in ascending key order              */
    int32_t grouped;     /* 1: hosts differ in GPU count; the table is stored count by count,
                          * each group in ascending key order                               */
    int64_t workspace_bytes;
    int32_t ranked;      /* 1: the ranked form is available (static_key and presorted): capacities and
                          * the host's rank in the order of Section 3.4.1 packed into one 64-bit
                          * value per host, compared with one subtraction per pair               */
    int32_t ranked_dropped_bits[4]; /* low bits of (GPUs, VRAM, millicpus, memory) the ranked form
                          * leaves out of its per-pair test; pairs that pass are re-tested exactly */
    int32_t reserved;
} nbos_snapshot_info;

/*
 * Launch shape for nbos_place_batch_ex. 0 in a field = choose automatically.
 *   lanes_per_request  1,2,4,8,16,32: lanes of one warp that share a request; each strides the
 *                      hosts and keeps its own best three, merged by xor-shuffles at the end.
 *   requests_per_lane  1,2,4,8: upper bound on requests one lane carries through the host loop.
 *   host_split         K >= 1: hosts are cut into K slices handled by different thread blocks;
 *                      K > 1 writes per-slice candidates to temporary device memory and runs a
 *                      merge kernel.
 *   tile_hosts         hosts per shared-memory tile (multiple of 32).
 *   grid_blocks        thread blocks along the request dimension (per host slice).
 *   pair_mode          how a (request, host) pair is evaluated when the snapshot has 32-bit keys:
 *                      0 = the fastest form the snapshot allows; 1 = four separate capacity
 *                      compares; 2 = packed capacity test with the key computed per pair (even if
 *                      the snapshot would allow ranking by the host part of the key alone);
 *                      3 = packed capacity test with the host part of the key compared per pair
 *                      (even if the table is stored in key order, where 0 drops that compare:
 *                      a feasible host then enters a request's best three exactly while the
 *                      request has fewer than three). Every form gives the same outputs.
 *   first_fit          1 = stop scanning a request's hosts at the third feasible one. Possible
 *                      when every host has the same key slope and the table is stored in key
 *                      order (nbos_snapshot_info: static_key and presorted), because then the
 *                      first three feasible hosts in table order are the best three; otherwise
 *                      the flag is ignored. Same outputs, far fewer (request, host) pairs looked
 *                      at: throughput of this variant is not a pairs/s figure.
 */
typedef struct nbos_launch_config {
    int32_t lanes_per_request;
    int32_t requests_per_lane;
    int32_t host_split;
    int32_t tile_hosts;
    int32_t grid_blocks;
    int32_t pair_mode;
    int32_t first_fit;
    int32_t reserved; /* must be 0 */
} nbos_launch_config;

/* Device bytes nbos_snapshot_create needs in `workspace` for this N and H (Section 3.4.1 state
 * turned into per-host records). Only n_snapshots, n_hosts and flags of `desc` are read. */
int nbos_snapshot_workspace_bytes(const nbos_snapshot_desc *desc, size_t *out_bytes);

/*
 * Build a snapshot from DEVICE arrays: validates, then derives one record per host -- the
 * largest GPU ask that passes the capacity test, the SR limit test of Section 3.4.1 and (if
 * asked) the idle test of Section 3.2.3, the three other capacities, and the two integers
 * (A, B) with  key(g) = A + g * B  that order hosts exactly as Section 3.4.1 does.
 *   workspace        DEVICE, 256-byte aligned, >= nbos_snapshot_workspace_bytes; caller-owned;
 *                    must stay valid and untouched until nbos_snapshot_destroy.
 *   arrays           DEVICE, 16-byte aligned.
 * Synchronises `cuda_stream` once (value-range validation needs a small read-back).
 * Errors: INVALID_ARG (NULL, alignment, N/H/R out of range, bad limit), RANGE (negative value,
 * C > G, G too large, key would not fit 63 bits), NO_MEMORY, CUDA, UNSUPPORTED_DEVICE.
 * On error *out is NULL and nothing is leaked.
 */
int nbos_snapshot_create(const nbos_snapshot_desc *desc, void *workspace, size_t workspace_bytes,
                         void *cuda_stream, nbos_snapshot **out);

/* Same operation from HOST arrays (any alignment). The library takes the workspace and a staging
 * buffer from a stream-ordered memory pool of its own (one per device, kept for the life of the
 * process so that repeated calls reuse the same memory) and gives them back to that pool in
 * nbos_snapshot_destroy / when the derivation has run. The host arrays have been read when the
 * call returns. */
int nbos_snapshot_create_host(const nbos_snapshot_desc *desc, void *cuda_stream,
                              nbos_snapshot **out);

/*
 * Refresh an existing snapshot from new cluster state of the same shape (same N, H, R, key order
 * and flags as at creation; `desc` carries the new arrays and limits): the per-host records of
 * Sections 3.2.1 / 3.4.1 are derived again with the key widths, packing layout and visiting-order
 * machinery chosen at creation. Unlike creation this reads nothing back and never synchronises:
 * it only queues work on `cuda_stream`, so a scheduler tick can queue "update, place, update,
 * place ..." without waiting. The price is that problems are reported late: if the new state
 * has a value outside the supported range, or does not fit the stored layout (more idle GPUs,
 * a larger subscription or capacity than the widths allow, a GPU count per host the snapshot did
 * not have), the device status word is raised, the tables and every placement made from them are
 * undefined, and nbos_snapshot_status returns NBOS_ERR_RANGE / NBOS_ERR_STALE_LAYOUT; destroy the
 * snapshot and create a new one then. A successful update clears what an earlier update reported;
 * a device-side wait that ran out (NBOS_ERR_DEVICE_TIMEOUT) stays reported until the snapshot is
 * destroyed.
 * The caller must make sure that no placement on ANOTHER stream is still using the snapshot;
 * work queued earlier on the same stream is ordered before the update.
 *   nbos_snapshot_update       arrays are DEVICE memory (16-byte aligned), read by the queued work
 *   nbos_snapshot_update_host  arrays are HOST memory; copied into device staging the library
 *                              keeps per device (two sets, taken in turn) on its copy-in stream,
 *                              in call order with the request copies of the host-buffer placement
 *                              calls; the derivation queued on `cuda_stream` waits for the copies.
 *                              Pageable arrays have been read when the call returns; PINNED arrays
 *                              are read asynchronously: keep them unchanged until `cuda_stream`
 *                              has reached the end of the update.
 * Errors at call time: INVALID_ARG (shape / flags differ, NULL or misaligned pointers, bad limit),
 * NO_MEMORY, CUDA.
 */
int nbos_snapshot_update(nbos_snapshot *snap, const nbos_snapshot_desc *desc, void *cuda_stream);
int nbos_snapshot_update_host(nbos_snapshot *snap, const nbos_snapshot_desc *desc, void *cuda_stream);

/* Frees the handle (and what nbos_snapshot_create_host allocated: that memory goes back to the
 * library's pool in the order of the stream the snapshot was created or last updated on). The
 * caller must make sure no nbos_place_batch on this snapshot is still running. NULL is accepted. */
int nbos_snapshot_destroy(nbos_snapshot *snap);

int nbos_snapshot_get_info(const nbos_snapshot *snap, nbos_snapshot_info *out);

/*
 * The placement decision of Sections 3.2.1 / 3.4.1 for a batch (definition at the top).
 *   requests   DEVICE [N * batch_per_snapshot * 4] int32, 16-byte aligned; request i of
 *              snapshot n at ((n * batch + i) * 4): GPUs, VRAM GB, millicpus, memory MB.
 *              A request with a negative field fits nowhere (all -1); that is not an error.
 *   out_hosts  DEVICE [N * batch * 3] int32: host indices (0 .. H-1) best first, -1 padding.
 *   out_found  DEVICE [N * batch] int32 or NULL: number of hosts found (0..3).
 * Asynchronous on `cuda_stream`; outputs are valid once the stream has been synchronised. The
 * snapshot is read-only here, so calls on different streams may overlap. batch == 0 is a no-op.
 * Errors: INVALID_ARG, CUDA, NO_MEMORY. A device-side wait that ran out is reported later by
 * nbos_snapshot_status.
 */
int nbos_place_batch(const nbos_snapshot *snap, const int32_t *requests, int64_t batch_per_snapshot,
                     int32_t *out_hosts, int32_t *out_found, void *cuda_stream);

/* Same, with an explicit launch shape (NULL = automatic). Every shape gives identical output. */
int nbos_place_batch_ex(const nbos_snapshot *snap, const int32_t *requests,
                        int64_t batch_per_snapshot, int32_t *out_hosts, int32_t *out_found,
                        void *cuda_stream, const nbos_launch_config *cfg);

/*
 * Same operation with HOST buffers (pinned memory makes the copies asynchronous and faster, but
 * any host memory works). The batch is cut into up to 4 chunks whose host-to-device copy, kernel
 * and device-to-host copy overlap on three internal streams (copies in, kernels, copies out;
 * created once per device, with two sets of device staging that successive calls take in turn and
 * that grow when a larger batch comes). The copies in start as soon as staging is free; the
 * kernels wait for the work queued on `cuda_stream` before the call (a snapshot update, say), and
 * `cuda_stream` in turn waits for the kernels, so that a later update of the snapshot queued on it
 * does not overtake them. Calls on the same device take their turns in the order they are made.
 *   nbos_place_batch_host        returns after the results are in the host buffers.
 *   nbos_place_batch_host_async  returns once the work is queued. Calls in a row overlap: the
 *                                copies in of one run beside the kernels of the one before and
 *                                the copies out of the one before that. The request and result
 *                                buffers belong to the library until nbos_place_batch_host_wait
 *                                (or a later nbos_place_batch_host on the same device) has
 *                                returned. With pageable host memory the copies block the caller
 *                                and nothing overlaps (still correct).
 *   nbos_place_batch_host_wait   blocks until every host-buffer call made so far on the
 *                                snapshot's device has delivered its results. Call it before
 *                                destroying a snapshot that asynchronous calls still use.
 * Errors: INVALID_ARG, NO_MEMORY, CUDA (after an error the internal streams are synchronised
 * before the call returns).
 */
int nbos_place_batch_host(const nbos_snapshot *snap, const int32_t *requests_host,
                          int64_t batch_per_snapshot, int32_t *out_hosts_host,
                          int32_t *out_found_host, void *cuda_stream);
int nbos_place_batch_host_async(const nbos_snapshot *snap, const int32_t *requests_host,
                                int64_t batch_per_snapshot, int32_t *out_hosts_host,
                                int32_t *out_found_host, void *cuda_stream);
int nbos_place_batch_host_wait(const nbos_snapshot *snap);

/*
 * Placement for callers that are not allowed to allocate device memory. (The paper has no
 * counterpart; this is a deployment variant of nbos_place_batch with the host-split launch
 * shape.)
 *
 * Who needs it: a scheduler that shares its GPU with a training or serving job which has
 * already handed all free device memory to its own pool, so that a cudaMalloc here can fail or
 * evict; and control loops with a latency budget, where the device-wide synchronisation and
 * the driver lock an allocation may take are not acceptable. nbos_place_batch allocates a
 * temporary candidate buffer whenever it cuts the hosts into slices (small batches against many
 * hosts). This entry point computes the same result with that buffer placed in a fixed array
 * of NBOS_NOALLOC_SCRATCH_BYTES that is part of the library image: every GPU on which the
 * library is loaded holds those bytes until the process exits. It calls no cudaMalloc,
 * cudaFree or other allocating routine. Inputs and outputs are still the caller's.
 *
 *   host_split   K, number of host slices (1..NBOS_NOALLOC_MAX_SPLIT; 0 = 4). It is lowered to
 *                what the host count allows. K = 1 uses no candidate buffer at all.
 *   limit        K * N * batch_per_snapshot * 3 keys (4 bytes each, 8 when the snapshot uses
 *                64-bit keys) must fit NBOS_NOALLOC_SCRATCH_BYTES; otherwise the call returns
 *                NBOS_ERR_NO_MEMORY, says so in nbos_last_error_detail(), and launches nothing.
 *   first call   The first call on each device looks up the array's device address
 *                (cudaGetSymbolAddress, with that device current). Make that first call during
 *                start-up, before any stream capture begins.
 *   sharing      All calls in the process, on all streams, use the same array, and it keeps
 *                whatever the previous call left. Nothing in it needs clearing: each call writes
 *                every slot it later reads. But two calls that overlap on the GPU (different
 *                streams, no dependency between them) race on it and give wrong results: order
 *                them on one stream or with events.
 * Other arguments, output and asynchrony as for nbos_place_batch; the snapshot must belong to
 * the current device.
 */
#define NBOS_NOALLOC_SCRATCH_BYTES (8u << 20)
#define NBOS_NOALLOC_MAX_SPLIT 64
int nbos_place_batch_noalloc(const nbos_snapshot *snap, const int32_t *requests,
                             int64_t batch_per_snapshot, int32_t *out_hosts, int32_t *out_found,
                             void *cuda_stream, int32_t host_split);

/*
 * Executor selection for a batch of cell executions (Section 3.2.2). When a cell is submitted,
 * the scheduler looks at the servers hosting the kernel's three replicas: a replica whose server
 * lacks the resources to run the cell now is told to yield, and with the resource information at
 * hand the scheduler designates the executor itself; if all three must yield, a replica has to
 * migrate (Section 3.2.3 -- find the target with nbos_place_batch on a snapshot created with
 * NBOS_REQUIRE_IDLE_GPUS and the idle capacities; its first column is the best target).
 *
 *   can run now   <=>  g,v,c,m >= 0 and G >= 1 and g <= G - C and v <= vram_gb and c <= millicpus
 *                      and m <= mem_mb  (pass the idle capacities). The SR limit is not tested:
 *                      the replica is already subscribed on its server.
 *   designated    =    among the replicas that can run, the first by (G - C descending,
 *                      S / (G * R) ascending -- compared exactly --, host index ascending, replica
 *                      slot ascending). The paper does not say which runnable replica is picked;
 *                      this is the default placement policy's order (Section 3.4.1).
 *
 *   state          DEVICE arrays [n_hosts] int32 of one cluster snapshot (not validated; a host
 *                  index outside 0..n_hosts-1 in replica_hosts, e.g. -1, means "no such replica")
 *   requests       DEVICE [n_kernels * 4] int32, 16-byte aligned: GPUs, VRAM GB, millicpus, MB
 *   replica_hosts  DEVICE [n_kernels * 3] int32 (any 4-byte alignment; when it is 16-byte aligned,
 *                  batches of 2^19 kernels and more are streamed through bulk asynchronous copies)
 *   out_executor   DEVICE [n_kernels] int32: host index of the designated executor, -1 = all yield
 *   out_can_run    DEVICE [n_kernels] int32: bit k set = the replica in slot k can run now
 * Asynchronous on `cuda_stream`; a per-call temporary of 36 bytes per host comes from the
 * library's stream-ordered pool. Errors: INVALID_ARG, NO_MEMORY, CUDA, UNSUPPORTED_DEVICE.
 */
typedef struct nbos_cluster_state {
    int32_t n_hosts;
    int32_t replicas_R;
    const int32_t *gpus_total, *gpus_subscribed, *gpus_committed;
    const int32_t *vram_gb, *millicpus, *mem_mb;
} nbos_cluster_state;

int nbos_select_executors(const nbos_cluster_state *state, const int32_t *requests,
                          const int32_t *replica_hosts, int64_t n_kernels, int32_t *out_executor,
                          int32_t *out_can_run, void *cuda_stream);

/*
 * Sequential placement with commits: the paper's scheduler places one kernel at a time, and a
 * placed kernel's replicas subscribe its GPUs on their three servers before the next kernel is
 * looked at (Sections 3.2.1, 3.4.1). For request i = 0, 1, ... of each snapshot, in order: the
 * same decision as nbos_place_batch against the current state; if three hosts were found, S of
 * each grows by the request's GPU count (its key and its remaining room under the SR limit move
 * accordingly); if fewer were found nothing changes (the kernel is not created). Committed GPUs
 * and the other capacities stay as they are. Snapshots are independent and run in parallel; the
 * snapshot object itself is not modified.
 *   snap            must have been created with NBOS_ROOM_FOR_COMMITS; at most
 *                   NBOS_SEQUENTIAL_MAX_HOSTS hosts (the evolving state lives on one SM up to
 *                   8,192 hosts, on the 2 to 8 SMs of a thread-block cluster beyond that);
 *                   otherwise INVALID_ARG / RANGE
 *   requests, out_hosts, out_found   as for nbos_place_batch
 *   out_subscribed  DEVICE [N * H] int32 or NULL: S of every host after the last request
 * Asynchronous on `cuda_stream`.
 */
#define NBOS_SEQUENTIAL_MAX_HOSTS 65536
int nbos_place_batch_sequential(const nbos_snapshot *snap, const int32_t *requests,
                                int64_t batch_per_snapshot, int32_t *out_hosts, int32_t *out_found,
                                int32_t *out_subscribed, void *cuda_stream);

/*
 * Cluster sums and the auto-scaler rule (Sections 3.4.1, 3.4.2), per snapshot:
 *   out_sums[4n + 0] = sum of G   (GPUs provisioned)
 *   out_sums[4n + 1] = sum of S   (GPUs subscribed; sum S / (sum G * R) is the cluster-wide SR)
 *   out_sums[4n + 2] = sum of C   (GPUs in active use)
 *   out_sums[4n + 3] = +1 if sum G < f * sum C   (capacity below the expected f * sum C: scale out)
 *                      -1 if f * sum C < sum G   (more provisioned than expected: servers may go)
 *                       0 if equal;   f = f_num / f_den, compared exactly (the paper uses 1.05 = 21/20)
 * Arrays: DEVICE [n_snapshots * n_hosts] int32 (not validated); out_sums: DEVICE [n_snapshots * 4]
 * int64. Asynchronous on `cuda_stream`.
 */
int nbos_cluster_sums(const int32_t *gpus_total, const int32_t *gpus_subscribed,
                      const int32_t *gpus_committed, int32_t n_snapshots, int32_t n_hosts,
                      int32_t f_num, int32_t f_den, int64_t *out_sums, void *cuda_stream);

/*
 * Scale-out deficit of a placed batch (Sections 3.2.1, 3.4.2: when fewer than three candidate
 * servers exist, as many additional servers as are missing get provisioned), per snapshot:
 *   out_deficit[2n + 0] = sum over the batch of (3 - found)
 *   out_deficit[2n + 1] = number of requests with found < 3
 * found: DEVICE [n_snapshots * batch_per_snapshot] int32 as written by nbos_place_batch;
 * out_deficit: DEVICE [n_snapshots * 2] int64. Asynchronous on `cuda_stream`.
 */
int nbos_scale_out_deficit(const int32_t *found, int32_t n_snapshots, int64_t batch_per_snapshot,
                           int64_t *out_deficit, void *cuda_stream);

/*
 * ---- Learned placement policies ------------------------------------------------------------------------
 * Section 3.2.1 calls the rule that ranks candidate servers a policy that can be replaced. A policy that is
 * learned scores every host for every request: a table of logits [rows, n_hosts], -inf where the host cannot
 * take the request. The entry points below train one on the exact rule's decisions (nbos_policy_distill),
 * keep it from sending everything to few hosts (nbos_policy_balance) and let it answer (nbos_policy_sample).
 * Read hosts as vocabulary entries or experts and rows as tokens and they are the same operators of a
 * language model.
 *
 *   data        DEVICE, aligned to its element type. Rows may start anywhere; those that start on 16-byte boundaries
 *               (data and row_stride) are the fastest.
 *   row_stride  elements from one row to the next, >= n_hosts (any value when rows <= 1)
 * All arithmetic is in 32 bits, with one rounding to the logits' type at the end: a row's sums over its hosts, and the balance
 * loss's sums over the rows that one block takes. That loss's sums over blocks and over hosts are in 64 bits; sampling adds
 * whole numbers. Results do not change from run to run: no floating-point atomics. Every call is asynchronous on
 * `cuda_stream`; temporaries come from the library's stream-ordered pool. rows == 0 is a no-op (outputs per group
 * are still written). Errors of all of them: INVALID_ARG, NO_MEMORY, CUDA, UNSUPPORTED_DEVICE.
 */
#define NBOS_F32 0
#define NBOS_BF16 1
#define NBOS_F16 2
#define NBOS_POLICY_MAX_ROWS 2147483647
#define NBOS_POLICY_MAX_K 256    /* hosts per row of a teacher / of a choice  */
#define NBOS_POLICY_MAX_DRAWS 8  /* hosts drawn per row by nbos_policy_sample */

typedef struct nbos_logits {
    const void *data;   /* DEVICE [rows][row_stride]              */
    int64_t rows;       /* 0 .. NBOS_POLICY_MAX_ROWS              */
    int64_t row_stride; /* elements                               */
    int32_t n_hosts;    /* 1 .. NBOS_MAX_HOSTS                    */
    int32_t dtype;      /* NBOS_F32 | NBOS_BF16 | NBOS_F16        */
} nbos_logits;

/*
 * Distillation from a teacher's k best hosts per row, forward and gradient.
 *   Entry j of row r counts if its host index is in 0..n_hosts-1 (-1 = no entry: what nbos_place_batch writes
 *   can be passed as it is), the row's logit x of that host is above -inf and its teacher logit t is above -inf.
 *     q = softmax over the row's counting entries of t / T          p = softmax over all hosts of x / T
 *     loss = T^2 * sum_j q_j (ln q_j - ln p[host_j])
 *     grad = T * (p - q scattered to its hosts) * grad_scale * grad_loss[r]
 *   A host that is listed twice counts with both entries. A row without a counting entry has loss 0 and gradient
 *   0. A NaN or +inf logit makes its row's loss and gradient NaN; a NaN teacher logit does not count.
 *   hosts           DEVICE [rows * k] int32
 *   teacher_logits  DEVICE float, row r at r * teacher_stride (0: the same k for every row); NULL = all equal
 *   temperature     T, finite and > 0
 *   grad_loss       DEVICE [rows] float, the gradient that arrives at the loss; NULL = 1
 *   out_loss        DEVICE [rows] float or NULL
 *   out_stats       DEVICE [rows * 2] float or NULL: (m, S), the row's largest logit and sum of e^((x - m) / T):
 *                   what nbos_policy_distill_backward needs. (-inf, 0) for a row of -inf.
 *   out_grad        DEVICE, the logits' type, rows grad_stride elements apart, or NULL (forward only). May be the
 *                   logits themselves (same stride); must not overlap them otherwise.
 * With out_grad the logits are read once for both directions. nbos_policy_distill_backward computes the same
 * gradient later, from the saved statistics.
 */
int nbos_policy_distill(const nbos_logits *logits, const int32_t *hosts, const float *teacher_logits,
                        int64_t teacher_stride, int32_t k, float temperature, const float *grad_loss,
                        float grad_scale, float *out_loss, float *out_stats, void *out_grad, int64_t grad_stride,
                        void *cuda_stream);
int nbos_policy_distill_backward(const nbos_logits *logits, const int32_t *hosts, const float *teacher_logits,
                                 int64_t teacher_stride, int32_t k, float temperature, const float *stats,
                                 const float *grad_loss, float grad_scale, void *out_grad, int64_t grad_stride,
                                 void *cuda_stream);

/*
 * Load-balance loss with per-host counts, forward and gradient. The rows are n_groups groups of rows / n_groups
 * (the snapshots of a what-if sweep, the sequences of a batch); each group has its own loss.
 *   hosts [rows * k]: the k hosts chosen per row, an index outside 0..n_hosts-1 (-1) = none. A row is live if it
 *   has at least one.
 *     count_h = how often host h was chosen in the group     f_h = count_h / sum of counts
 *     P_h     = mean over the group's live rows of softmax(x)_h
 *     loss    = n_hosts * sum_h f_h P_h                      (1 when either is uniform)
 *     grad    = n_hosts / live * p_h (f_h - sum_i f_i p_i) * grad_scale * grad_loss[group]; 0 for other rows
 *   f is a constant for the gradient (it is a count). A group without a live row has loss, shares and gradient
 *   0. A live row of -inf adds nothing to P and has gradient 0. NaN and +inf logits make their row's gradient, and
 *   their group's loss and P, NaN.
 *   out_loss    DEVICE [n_groups] float
 *   out_counts  DEVICE [n_groups * n_hosts] int32
 *   out_shares  DEVICE [n_groups * n_hosts] float (P) or NULL
 *   out_stats   DEVICE [rows * 2] float or NULL: (m, S) per row as above with T = 1, for the backward call; not
 *               written for rows that are not live
 *   out_grad    as above. f depends on the choices alone, so one pass over the logits gives both directions.
 * rows * k and rows / n_groups * k must fit in 31 bits; rows must be a multiple of n_groups.
 */
int nbos_policy_balance(const nbos_logits *logits, int32_t n_groups, const int32_t *hosts, int32_t k,
                        const float *grad_loss, float grad_scale, float *out_loss, int32_t *out_counts,
                        float *out_shares, float *out_stats, void *out_grad, int64_t grad_stride,
                        void *cuda_stream);
int nbos_policy_balance_backward(const nbos_logits *logits, int32_t n_groups, const int32_t *hosts, int32_t k,
                                 const float *stats, const float *grad_loss, float grad_scale, void *out_grad,
                                 int64_t grad_stride, void *cuda_stream);

/*
 * Sampling distinct hosts from given random numbers. Per row, with m the largest logit:
 *   weight   w_h = floor(2^31 * 2^((x_h - m) * c)), c = float(log2 e) / T, each step in 32-bit floats, 2^y as
 *            exp2f. A whole number: sums of weights are exact and do not depend on the order they are taken in.
 *   filters  in the order (x descending, index ascending) keep a first part of the hosts:
 *              top-k  the first top_k;  <= 0 = off
 *              top-p  of those, each host before which less than max(1, floor(A * floor(p * 2^24) / 2^24))
 *                     of weight stands, A the weight of the top-k hosts;  p >= 1 or NaN = off
 *              min-p  of those, hosts with w >= floor(min_p * 2^31);  <= 0 or NaN = off
 *   draw d   t = floor(A' * floor(u_d * 2^24) / 2^24), A' the weight left; the lowest host index at which the running
 *            sum of weights (in index order) exceeds t; its weight is then taken out. -1 once no weight is left.
 *   T <= 2^-20 or NaN keeps the best host alone (greedy). A NaN logit counts as -inf, +inf as the largest
 *   finite float. u is clamped to [0, 1 - 2^-24], NaN counts as 0.
 *   uniforms     DEVICE [rows * draws] float
 *   temperature, top_p, min_p  DEVICE [rows] float or NULL (1 / off / off);  top_k  DEVICE [rows] int32 or NULL
 *   draws        1 .. NBOS_POLICY_MAX_DRAWS (three for the replicas of a kernel, one for a token)
 *   out_hosts    DEVICE [rows * draws] int32, in the order drawn, -1 padding
 *   out_found    DEVICE [rows] int32 or NULL: how many were drawn
 */
int nbos_policy_sample(const nbos_logits *logits, const float *uniforms, const float *temperature,
                       const int32_t *top_k, const float *top_p, const float *min_p, int32_t draws,
                       int32_t *out_hosts, int32_t *out_found, void *cuda_stream);

/*
 * Distillation of a two-tower policy without its table of logits. Such a policy scores a host for a request as the
 * product of two vectors; with many requests and hosts the table [rows, n_hosts] is far larger than the vectors, and is
 * never stored here: the forward call keeps a row's maximum and sum (and the scores at its hosts; more than four a row are sorted first, 4
 * bytes each), the backward call computes the scores once more and holds
 * pieces of about 512 MB (or 256 rows / hosts, where that is more) of their gradient.
 *   x[g, r, h] = sum_i requests[g, r, i] * hosts[g, h, i], -inf unless the request fits the host: asks[g, r, i] <= room[g, h, i] and
 *   asks[g, r, i] >= 0 for all four i. (With asks = the requests of nbos_place_batch and room[0] = the GPUs that the host's size and
 *   subscription limit leave, that is the rule's own test.) asks and room NULL: every request fits every host.
 * Loss and gradient are those of nbos_policy_distill on these logits, row by row and entry by entry; rows that fit nowhere, or
 * without a counting entry, have loss and gradient 0. (A vector that is not finite may make the other tower's gradient NaN,
 * also where none of its scores counts: 0 times it is not 0.)
 *     grad_requests = G hosts, grad_hosts = G^T requests, G = T * (p - q) * grad_scale * grad_loss[r]
 * Products are of 16-bit values with 32-bit sums, statistics are in 32 bits. Before it is multiplied, G gets a factor that brings the
 * largest finite |grad_loss| of a row that counts to just below a power of two (2^15 in 16-bit floats), and each entry is held as two
 * values of the vectors' type, the second what the first's rounding took off; a gradient is rounded once at the end. In 16-bit floats
 * a row whose grad_loss is 2^-n of the largest keeps its p down to 2^(n - 29) in full and to 2^(n - 39) in part. With gradient_values = 1 an
 * entry is one value: the backward call is 1.8 times as fast where products bound it, and its gradients are off as G's rounding makes
 * them, by up to 2^-8 (bf16) or 2^-11 (f16) of each term's size, which is much where a row's terms cancel (vectors with a large part in common).
 *   towers          vectors DEVICE, NBOS_BF16 or NBOS_F16, of any alignment and row stride >= width; rows on 16-byte boundaries (address,
 *                   strides) are read as they lie, others are copied first. A group stride may be 0 (one table for all groups).
 *   hosts, teacher_logits, teacher_stride, k, temperature, grad_loss, grad_scale   as for nbos_policy_distill; hosts
 *                   [n_groups * rows * k]
 *   out_loss        DEVICE [n_groups * rows] float or NULL
 *   out_stats       DEVICE [n_groups * rows * (2 + k)] float or NULL: what the backward call needs (a row's m and S, or (0, inf) if it
 *                   has no counting entry, and its logits at its hosts, -inf where the entry is none or does not fit)
 *   out_grad_*      DEVICE, the vectors' type, or NULL; groups must not overlap; may not overlap the inputs
 * The kernels wait on copies and products with a limit; nbos_policy_towers_status synchronises `cuda_stream` and returns
 * NBOS_ERR_DEVICE_TIMEOUT, once, if a wait on the current device ran out since it was last asked. Until it is asked, losses and
 * gradients are NaN (those of the call whose wait ran out at least where they are missing), statistics undefined.
 */
#define NBOS_POLICY_MAX_WIDTH 65536
typedef struct nbos_towers {
    const void *requests;         /* DEVICE [n_groups][rows][request_stride]    */
    const void *hosts;            /* DEVICE [n_groups][n_hosts][host_stride]    */
    int64_t rows;                 /* per group; n_groups * rows < 2^31          */
    int64_t request_stride, request_group_stride, host_stride, host_group_stride; /* elements */
    int32_t n_groups;             /* 1 .. 65535 (the snapshots of a sweep)      */
    int32_t n_hosts;              /* 1 .. NBOS_MAX_HOSTS                        */
    int32_t width;                /* 1 .. NBOS_POLICY_MAX_WIDTH                 */
    int32_t dtype;                /* NBOS_BF16 | NBOS_F16                       */
    const int32_t *asks;          /* DEVICE [n_groups * rows * 4] or NULL, 16-byte aligned    */
    const int32_t *room;          /* DEVICE [n_groups * n_hosts * 4] or NULL, 16-byte aligned */
    int32_t gradient_values;      /* backward: 16-bit values that hold an entry of G: 2, or 1; 0: 2 */
} nbos_towers;

int nbos_policy_towers(const nbos_towers *towers, const int32_t *hosts, const float *teacher_logits,
                       int64_t teacher_stride, int32_t k, float temperature, float *out_loss, float *out_stats,
                       void *cuda_stream);
int nbos_policy_towers_backward(const nbos_towers *towers, const int32_t *hosts, const float *teacher_logits,
                                int64_t teacher_stride, int32_t k, float temperature, const float *stats,
                                const float *grad_loss, float grad_scale, void *out_grad_requests,
                                int64_t grad_request_stride, int64_t grad_request_group_stride, void *out_grad_hosts,
                                int64_t grad_host_stride, int64_t grad_host_group_stride, void *cuda_stream);
int nbos_policy_towers_status(void *cuda_stream);

/*
 * The norms around a residual block of a policy's tower: after its branch, with a gate, onto the scaled residual, and before the
 * next block, in one pass. Row by row, with norm(v) = v / sqrt(mean(v^2) + eps):
 *     r = residual_scale * residual + gate * (norm(branch) * post_weight)        out_residual
 *     h = norm(r) * pre_weight                                                   out_normed
 * h is of the unrounded r; everything is in 32 bits (whose squares overflow beyond 1.8e19) and rounded once.
 *   residual, branch   DEVICE [rows], row_stride >= width apart, aligned to their type; tables whose rows all start on 16-byte
 *                      boundaries are the fastest
 *   gate               DEVICE or NULL (1): row r uses gate row r / rows_per_gate: 1 = a gate for each row, rows per group = one for
 *                      each group, rows = one for all. rows must be a multiple.
 *   post_weight, pre_weight  DEVICE [width] or NULL (1)
 *   gate_dtype, weight_dtype  dtype or NBOS_F32 each; gradients have the same
 *   out_residual, out_normed  DEVICE, dtype, or NULL; may be residual or branch themselves (same stride), must not overlap any input
 *                      otherwise
 *   out_stats          DEVICE [rows * 2] float or NULL: 1 / sqrt(mean + eps) of both norms, for the backward call
 * Backward: grad_residual is what arrives at out_residual, grad_normed at out_normed (either may be NULL: 0). Any of the outputs may
 * be NULL. out_grad_residual and out_grad_branch may be grad_residual or grad_normed themselves (same stride). Gradients of weights
 * and of shared gates are sums over rows in 32 bits, in an order that does not change from run to run.
 */
#define NBOS_BLOCK_MAX_WIDTH 16384
typedef struct nbos_block {
    const void *residual, *branch, *gate, *post_weight, *pre_weight;
    int64_t residual_stride, branch_stride, gate_stride; /* elements */
    int64_t rows;          /* 0 .. NBOS_POLICY_MAX_ROWS */
    int64_t rows_per_gate; /* >= 1 where there is a gate */
    int32_t width;         /* 1 .. NBOS_BLOCK_MAX_WIDTH */
    int32_t dtype, gate_dtype, weight_dtype;
    float residual_scale;  /* finite       */
    float eps;             /* finite, >= 0 */
} nbos_block;

int nbos_policy_block_norm(const nbos_block *block, void *out_residual, int64_t out_residual_stride, void *out_normed,
                           int64_t out_normed_stride, float *out_stats, void *cuda_stream);
int nbos_policy_block_norm_backward(const nbos_block *block, const float *stats, const void *grad_residual,
                                    int64_t grad_residual_stride, const void *grad_normed, int64_t grad_normed_stride,
                                    void *out_grad_residual, int64_t out_grad_residual_stride, void *out_grad_branch,
                                    int64_t out_grad_branch_stride, void *out_grad_gate, int64_t out_grad_gate_stride,
                                    void *out_grad_post, void *out_grad_pre, void *cuda_stream);

/*
 * The global norm over many tensors (the gradients of a policy), and clipping by it:
 *     norm = (sum over all values of x^2)^(1/2) [NBOS_NORM_2] or max |x| [NBOS_NORM_INF]
 *     out  = x * min(1, max_norm / (norm + 1e-6)), rounded once to the tensor's type
 * Squares are summed in 32 bits within 64 bytes of values of a thread (16 or 32), where that neither overflows nor loses small values, and in 64 bits
 * beyond and otherwise; the sums do not change from run to run. (A norm beyond 32 bits is written as infinity, and
 * clips by its true value.) A NaN makes the norm and every output NaN; an infinity makes the norm infinite and, at a finite max_norm,
 * finite values 0 and itself NaN (as the formula says). No tensors, or none with values: norm 0.
 *   data, numel, dtype  HOST arrays [n_tensors]: DEVICE address (aligned to its type), number of values (0 .. 2^40, contiguous) and
 *                       NBOS_* type of each tensor; types may be mixed
 *   out                 HOST array [n_tensors] of DEVICE addresses, or NULL: the norm alone. An output may be its own input (nothing is
 *                       written then when there is nothing to clip); it must not overlap any tensor otherwise.
 *   max_norm            >= 0; infinity clips nothing (a NaN among the values still makes all of them NaN)
 *   out_norm            DEVICE float or NULL
 * The host arrays have been read when the call returns. Asynchronous on `cuda_stream`.
 */
#define NBOS_NORM_2 0
#define NBOS_NORM_INF 1
int nbos_policy_clip(const void *const *data, void *const *out, const int64_t *numel, const int32_t *dtype,
                     int32_t n_tensors, float max_norm, int32_t norm_kind, float *out_norm, void *cuda_stream);

/* Synchronises `cuda_stream` and returns the sticky device status of this snapshot: NBOS_OK, or
 * NBOS_ERR_DEVICE_TIMEOUT if some kernel gave up on a bounded wait (its outputs are then
 * undefined), NBOS_ERR_RANGE / NBOS_ERR_STALE_LAYOUT after an nbos_snapshot_update whose new state
 * was invalid / did not fit the snapshot's layout. */
int nbos_snapshot_status(const nbos_snapshot *snap, void *cuda_stream);

const char *nbos_strerror(int status);
const char *nbos_last_error_detail(void);

#ifdef __cplusplus
}
#endif
#endif /* NBOS_H_ */
