/*
 * libivf -- IVF-Flat nearest-neighbour search with lookahead prefetch for one
 * MI355X (gfx950).  C ABI: plain pointers and sizes, no C++ or torch types.
 *
 * The operations are those of TeleRAG (arxiv 2502.20969):
 *   - IVF search (App. B): coarse scoring of the query against all centroids,
 *     selection of the nprobe nearest clusters, a scan of the rows of those
 *     clusters, and the k nearest rows.
 *   - Lookahead retrieval (Sec. 4.1 steps 1-4, Sec. 4.3 "Prefetching target"):
 *     clusters ranked by q_in are copied host->device under a byte budget while
 *     other work runs; q_out is then searched over the resident clusters
 *     (C_overlap) on the GPU and over the others (C_miss) on the host, and the
 *     two partial results are merged.
 *
 * Conventions
 *   - Every function returns 0 (IVF_OK) or a negative ivf_status; nothing
 *     throws or aborts across this boundary.  ivf_strerror() names a status;
 *     ivf_last_error() gives a longer message for the calling thread.
 *   - "host" pointers are ordinary process memory unless "pinned" is said;
 *     "device" pointers are HIP device memory on the current device.
 *   - An index is used by one host thread at a time.  The library never frees
 *     or keeps caller memory unless a function says the index adopts it.
 *   - Metric (App. B, the distance d): IVF_IP ranks by inner product, larger is
 *     nearer, reported distances are the raw inner products (descending).
 *     IVF_L2 ranks by squared Euclidean distance, smaller is nearer, reported
 *     distances are the squared distances (ascending).  The coarse and the fine
 *     stage use the same metric.
 *   - Order: equal scores are ordered by smaller cluster index (coarse stage)
 *     or smaller vector id (fine stage), so results are deterministic.
 *   - nprobe larger than nlist is clamped to nlist.  When fewer than k rows
 *     were scanned the tail is padded with id -1 and distance -INF (IP) or
 *     +INF (L2).
 *   - Arithmetic: coarse scores are accumulated in fp64.  The list scan
 *     accumulates in fp32 over rows stored as fp32 / fp16 / bf16 with the fp32
 *     query; the k' = k + max(8, k / 8) best rows are then re-scored in fp64 and
 *     ordered by that score, and the fp64 value rounded to fp32 is what is
 *     returned.  The k nearest are exact with respect to the fp64 scores: when
 *     the k-th fp64 score found is not above the last fp32 score kept by more
 *     than a bound of the scan's rounding, a row that was dropped could belong
 *     to the result, and the query gets an exact second pass (every selected
 *     row scored in fp64) on the device, and likewise on the host for the host
 *     part of a hybrid search.
 */
#ifndef IVF_H
#define IVF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ivf_index ivf_index; /* opaque */

enum ivf_status {
    IVF_OK = 0,
    IVF_EINVAL = -1, /* bad argument: NULL, size < 1, unknown enum, assignment out of range */
    IVF_ENOMEM = -2, /* host or device allocation failed; the index is unchanged */
    IVF_EHIP = -3,   /* a HIP call failed; ivf_last_error() holds its text */
    IVF_ESTATE = -4, /* call not valid for this index (e.g. prefetch on a device-resident index) */
    IVF_ELIMIT = -5  /* a size is above what this build supports (k, d, n) */
};

enum ivf_metric { IVF_IP = 0, IVF_L2 = 1 };
enum ivf_dtype { IVF_F32 = 0, IVF_F16 = 1, IVF_BF16 = 2 }; /* storage type of list rows */
enum ivf_placement {
    IVF_PLACE_DEVICE = 0, /* every list resident in HBM */
    IVF_PLACE_HOST = 1    /* lists in pinned host memory + a device prefetch buffer
                             (Sec. "Implementation Details": pinned region, fixed GPU buffer) */
};

#define IVF_PREFETCH_RESET 1u /* drop all residency before planning (each request starts cold) */

#define IVF_MAX_K 112 /* largest k of ivf_search / ivf_search_device */

typedef struct ivf_prefetch_stats {
    int32_t n_ranked;   /* clusters considered (sum over queries of min(nprobe, nlist)) */
    int32_t n_taken;    /* clusters whose copy was enqueued by this call */
    int32_t n_skipped;  /* clusters that did not fit the remaining budget or buffer */
    int32_t n_resident; /* clusters considered that were already resident */
    uint64_t bytes;     /* payload bytes enqueued by this call */
    uint64_t buffer_used; /* bytes of the device buffer in use after this call */
} ivf_prefetch_stats;

typedef struct ivf_search_stats {
    int32_t n_probed;      /* sum over queries of clusters selected */
    int32_t n_overlap;     /* of those, scanned on the GPU */
    int32_t n_miss;        /* of those, scanned on the host */
    float hit_rate;        /* mean over queries of |C_overlap| / |C_out| (Table 1 caption) */
    uint64_t bytes_gpu;    /* list bytes the GPU scan covered: sum n_c*d*elem over C_overlap */
    uint64_t bytes_host;   /* list bytes the host scan covered */
    float ms_total;        /* wall time of the call */
    float ms_probe;        /* until the selected clusters were known to the host (host placement) */
    float ms_host_scan;    /* host scan of C_miss */
    int32_t n_exact_gpu;   /* queries whose GPU part needed the exact second pass (see "Arithmetic" above) */
    int32_t n_exact_host;  /* queries whose host part needed it */
} ivf_search_stats;

typedef struct ivf_profile {
    uint64_t calls;        /* searches measured since ivf_profile_reset() */
    double ms_coarse;      /* summed HIP-event time of the coarse-scoring kernel */
    double ms_select;      /* ... of the top-nprobe selection kernels; none where the scan selects the clusters itself */
    double ms_scan;        /* ... of the list-scan kernel, with the selection where it does that */
    double ms_merge;       /* ... of the merge / re-score kernel */
    uint64_t scan_bytes;   /* summed list bytes the scan kernels covered */
    uint64_t scan_rows;    /* summed rows the scan kernels covered */
} ivf_profile;

/*
 * Builds cluster-major lists from rows in input order (one-time; the a0 step:
 * the contiguous cluster-major region of Sec. "Implementation Details").
 *   vectors    host, n x d row-major in `dtype`
 *   centroids  host, nlist x d float32, copied to the device
 *   assign     host, n entries in [0, nlist): the list of each row
 *   ids        host, n entries >= 0, or NULL for ids 0..n-1
 *   device_buffer_bytes  size of the prefetch buffer (IVF_PLACE_HOST only)
 *   compute_stream, copy_stream  hipStream_t values, or NULL for streams the
 *              library creates; kernels run on the first, prefetch copies on
 *              the second; both must be of default priority
 * Rows keep their input order inside a list.  The library owns all storage it
 * creates (device lists, or a pinned host region for IVF_PLACE_HOST).
 */
int ivf_build_layout(const void* vectors, int64_t n, int32_t d, int dtype,
                     const float* centroids, int32_t nlist, const int32_t* assign,
                     const int64_t* ids, int metric, int placement,
                     size_t device_buffer_bytes, void* compute_stream, void* copy_stream,
                     ivf_index** out);

/*
 * Adopts rows that are already cluster-major, without copying them.
 *   lists      IVF_PLACE_DEVICE: device pointer; IVF_PLACE_HOST: pinned host pointer
 *              (allocated with hipHostMalloc, e.g. a torch pinned tensor).  Owned by the
 *              caller and must outlive the index.
 *   offsets    host, nlist + 1 entries: list c = rows offsets[c] .. offsets[c+1]
 *   ids        host, n entries >= 0, or NULL for ids = row position
 */
int ivf_adopt_layout(void* lists, const int64_t* offsets, const int64_t* ids, int64_t n,
                     int32_t d, int dtype, const float* centroids, int32_t nlist, int metric,
                     int placement, size_t device_buffer_bytes, void* compute_stream,
                     void* copy_stream, ivf_index** out);

void ivf_free(ivf_index* index);

/*
 * Lookahead step 1 (Sec. 4.1 "Predict & prefetch", Sec. 4.3 "Prefetching target").
 * For each of the nq queries q_in (host, nq x d float32): ranks all clusters, walks the
 * nprobe nearest in order and enqueues on copy_stream the copy of every cluster that is
 * not resident and fits both the remaining budget (budget_bytes / nq per query) and the
 * remaining device buffer; a cluster that does not fit is skipped whole and the walk goes
 * on.  A cluster's size is n_c * d * element size.  Returns once the copies are enqueued;
 * the next ivf_search waits for them on the device.  IVF_PLACE_HOST only.
 */
int ivf_prefetch(ivf_index* index, const float* q_in, int32_t nq, int32_t nprobe,
                 size_t budget_bytes, uint32_t flags, ivf_prefetch_stats* stats /* or NULL */);

/* Blocks the host until all enqueued prefetch copies have finished; *ms (or NULL) receives
 * the HIP-event time from the first to the last copy of the most recent ivf_prefetch. */
int ivf_prefetch_wait(ivf_index* index, float* ms);

/*
 * IVF search (App. B; with host placement: Sec. 4.1 steps 2-4).
 *   q_out  host, nq x d float32      ids    host, nq x k, nearest first
 *   dists  host, nq x k float32
 * On return the outputs are complete (for nq = 1 the call returns as soon as the last kernel
 * has published them; work enqueued later on compute_stream is ordered behind that kernel).
 * With IVF_PLACE_HOST the clusters selected for
 * q_out that are resident are scanned on the GPU while the others are scanned by host
 * threads; the result equals a search with every list resident.
 */
int ivf_search(ivf_index* index, const float* q_out, int32_t nq, int32_t nprobe, int32_t k,
               int64_t* ids, float* dists, ivf_search_stats* stats /* or NULL */);

/*
 * The same search with device-resident queries and outputs (all device pointers), enqueued
 * on compute_stream without waiting: outputs are complete once that stream has reached
 * this point (with a pipeline depth above 1: see ivf_set_pipeline_depth; searched list-major:
 * see ivf_set_batch_mode, after ivf_synchronize()).  q_dev must be 16-byte aligned; q_dev, ids_dev
 * and dists_dev must stay valid until the outputs are complete.  IVF_PLACE_DEVICE only.  nq, nprobe and k must not exceed what
 * ivf_reserve() or an earlier search (in the same batch mode) has sized the workspace for, else the call
 * sizes it itself, which synchronises the device.
 */
int ivf_search_device(ivf_index* index, const float* q_dev, int32_t nq, int32_t nprobe,
                      int32_t k, int64_t* ids_dev, float* dists_dev);

/* Sizes the workspace for searches up to (nq, nprobe, k) so that later calls allocate nothing (a list-major
 * batch of rows whose d is a multiple of 64 sizes more of it in the first such call).  List-major batches need
 * about 530 KB per query and lane beside what the rows themselves take; over rows of other widths, where they
 * are searched in slices, for at most 4096 queries (2.2 GB), and only when a batch of up to these sizes may be
 * searched so. */
int ivf_reserve(ivf_index* index, int32_t nq, int32_t nprobe, int32_t k);

/* Bounds the device memory that the list-major workspace of each lane may take (default: no bound) and gives
 * back what it holds; waits for the device.  What does not fit: over rows whose d is a multiple of 64 a
 * list-major batch fails with IVF_ENOMEM, as when the device has no more memory; over rows of other widths the
 * batch is searched in smaller slices, or query by query when not even four queries fit.  Like every call that
 * sizes the workspace anew it leaves list-major calls that were captured into a graph without theirs. */
int ivf_limit_batch_memory(ivf_index* index, size_t bytes);

/*
 * ivf_search_device for callers that cannot allocate: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and same results as a
 * query-by-query ivf_search_device, enqueued on compute_stream, but the workspace (coarse scores,
 * selected clusters and their tables, the scan wavefronts' candidate lists, the flags and lists of
 * the exact second pass) lives in one fixed
 * device array of IVF_NOALLOC_SCRATCH_BYTES that the library holds on every GPU it runs on until
 * the process ends.  The call allocates and frees nothing, on the host side of HIP or on the device.
 *   - A search whose workspace does not fit (roughly nq x (8 nlist + 32 nprobe) + 2100 x grid x nq
 *     bytes for k <= 56, twice the second term above that, grid <= 2 x compute units per query and
 *     fewer per query when nq is large: one query of a 1024-list index needs 1.1 MB) is refused with
 *     IVF_ELIMIT and nothing is enqueued.
 *   - Always query by query (the batch mode and the pipeline depth are ignored).  IVF_PLACE_DEVICE only.
 *   - Every call on a GPU shares that GPU's array, also across indexes: calls whose kernels could
 *     overlap on one GPU (other streams, other threads) race.  Calls on one compute_stream are
 *     ordered by the stream.  IVF_ESTATE while a list-major ivf_search_device batch is unfinished.
 */
#define IVF_NOALLOC_SCRATCH_BYTES (8u << 20)
int ivf_search_device_noalloc(ivf_index* index, const float* q_dev, int32_t nq, int32_t nprobe,
                              int32_t k, int64_t* ids_dev, float* dists_dev);

/*
 * Overlap of independent searches (batch-1 serving: one query's coarse scoring, selection and
 * merge run on a few compute units while another query's scan streams its lists).  With depth
 * n > 1, successive ivf_search_device calls rotate over n internal streams (the first is
 * compute_stream), each with its own workspace; inputs must be complete when the call is made,
 * and outputs are complete after ivf_synchronize() (which also runs the exact second pass for
 * the queries that need it; with depth 1 that pass follows every search on the stream).  List-major batches overlap in the same way
 * (the kernels that prepare one batch run beside the scan of the one before).  Depth 1 (the
 * default) keeps everything on compute_stream.  Changing the depth synchronises the device.  IVF_PLACE_DEVICE only; depth
 * in [1, 16].
 */
int ivf_set_pipeline_depth(ivf_index* index, int32_t depth);
/* Blocks the host until every search enqueued by ivf_search_device has finished. */
int ivf_synchronize(ivf_index* index);

/*
 * How a call with several queries is executed (Sec. 4.2 "Batching").
 *   0  automatic: batches of 4 or more queries on an index that has the list-major path are
 *      searched list-major (each selected cluster is read once per group of up to 32 queries,
 *      16 of fp32 rows, that probe it), unless they are so small that query by query is faster
 *      (bytes_gpu counts each cluster once all the same, as the list-major search does that such a
 *      batch may also get).  So are batches that are expected to gain by it on a device-resident index whose d
 *      is no multiple of 64, but these behave like a query-by-query call in every respect: outputs
 *      of ivf_search_device are complete in stream order, bytes_gpu counts every query's clusters,
 *      and a call under stream capture is enqueued query by query.  Anything else query by query
 *   1  always query by query
 *   2  list-major from 2 queries on; IVF_ESTATE (and the mode stays) when the index has no
 *      list-major path, rows whose d is no multiple of 64 among them
 * An index has the list-major path when all its rows are in HBM (IVF_PLACE_DEVICE), there are
 * fewer than 2^32 of them, and d is a multiple of 64 whose group of queries (32 of fp16 / bf16, 16
 * of fp32) fits LDS; any storage type, both metrics.  (The scan itself reads rows of any width from 16
 * bytes on; batches of those are completed in another way and belong to mode 0.)
 * The results are the same in every mode (the MFMA scores only filter rows; the ranking uses
 * fp64 re-scores with the fp32 query).  A list-major batch may leave a few queries to be
 * searched again one by one (their candidate lists overflowed): ivf_search does that before it
 * returns; ivf_search_device returns without waiting and the library finishes the batch when
 * its stream is next needed or in ivf_synchronize(), so the outputs of a list-major
 * ivf_search_device call are complete after ivf_synchronize() only, and q_dev, ids_dev and
 * dists_dev must stay valid until then.  With bytes_gpu of ivf_search_stats a list-major call
 * reports the bytes of the union of the selected clusters.
 */
int ivf_set_batch_mode(ivf_index* index, int32_t mode);

/* Stage-level entry points, used by the parity tests. */
/* coarse scores of App. B's first step: scores (host, nq x nlist fp64), raw metric values */
int ivf_coarse_scores(ivf_index* index, const float* q, int32_t nq, double* scores);
/* the nprobe nearest clusters, nearest first: clusters (host, nq x min(nprobe, nlist)) */
int ivf_probe(ivf_index* index, const float* q, int32_t nq, int32_t nprobe, int32_t* clusters);
/*
 * The scores the list-major scan filters with (Sec. 4.2 "Batching": the matrix-matrix product), for
 * every row of one cluster against nq <= 32 queries: scores (host, nq x rows of the cluster, in row
 * order) are the filter scores, larger is better: the products of the matrix cores, or of the vector units for up
 * to 8 queries and fp32 rows (query rounded to the
 * storage type, fp32 accumulation) for the inner product, 2 <q, y> - |y|^2 - |q|^2 from the same
 * products and the stored row norms for squared L2; eps (host, nq) is the bound the scan
 * assumes for |score - exact value| (exact: <q, y>, or -|q - y|^2, with the fp32 query).
 * Only for an index that has the list-major path or that automatic mode searches list-major (see
 * ivf_set_batch_mode), clusters of at most 65536 rows.
 */
int ivf_batched_scores(ivf_index* index, const float* q, int32_t nq, int32_t cluster, float* scores, float* eps);
/* how the most recent ivf_prefetch copies its clusters: by_kernel of them with one kernel that reads the pinned lists,
 * by_engine with one engine copy each (either may be NULL; empty clusters count for neither) */
int ivf_prefetch_ways(const ivf_index* index, int32_t* by_kernel, int32_t* by_engine);
/* resident clusters in ascending order; *n in: capacity of clusters, out: count */
int ivf_resident(ivf_index* index, int32_t* clusters, int32_t* n);
/* layout as built: offsets (host, nlist + 1) and/or ids (host, n); either may be NULL */
int ivf_get_layout(ivf_index* index, int64_t* offsets, int64_t* ids);
/*
 * The plan of ivf_prefetch on its own (Sec. 4.3 "Prefetching target", Sec. 4.2 "Batching"): the
 * budget walk over clusters that are already ranked.  Needs no index and no GPU; ivf_prefetch runs
 * the same code after ranking on the GPU.
 *   ranked        host, nq x nprobe cluster numbers, nearest first for each query
 *   offsets       host, nlist + 1 row offsets; a cluster's size is its rows x row_bytes
 *   resident_off  host, nlist entries, in/out: row offset of a resident cluster in the buffer, -1 = absent
 *   *buffer_used  in/out: bytes of the buffer in use (clusters are placed at this mark)
 *   taken         host, room for nq x nprobe entries: the clusters to copy, in order; *n_taken = count
 * stats (or NULL) as ivf_prefetch fills it.
 */
int ivf_prefetch_plan(const int32_t* ranked, int32_t nq, int32_t nprobe, const int64_t* offsets,
                      int32_t nlist, size_t row_bytes, size_t budget_bytes, size_t buffer_bytes,
                      int64_t* resident_off, size_t* buffer_used, int32_t* taken, int32_t* n_taken,
                      ivf_prefetch_stats* stats /* or NULL */);
/*
 * The host part of ivf_cache_end_round on its own (Sec. 4.2 "Cache design"), after the hotness
 * update: which clusters leave and how the survivors are moved.  Needs no index and no GPU;
 * ivf_cache_end_round runs the same code and then performs the moves with device copies.
 *   hotness       host, nlist float32, in/out: evicted clusters get -1
 *   resident_off  host, nlist, in/out: row offset in the buffer, -1 = not cached
 *   *buffer_used  in/out: bytes in use
 *   evicted       host, room for nlist entries, in the order the clusters leave; *n_evicted = count
 *   moves         host, room for nlist entries, in the order to carry them out; *n_moves = count.
 *                 A move copies `bytes` bytes from from_byte to to_byte of the buffer; via_staging = 1
 *                 when source and destination overlap (copy out to a staging area first).
 */
typedef struct ivf_cache_move {
    int32_t cluster;
    int32_t via_staging;
    uint64_t from_byte, to_byte, bytes;
} ivf_cache_move;
int ivf_cache_plan(float* hotness, const int64_t* offsets, int32_t nlist, size_t row_bytes,
                   int64_t* resident_off, size_t* buffer_used, size_t buffer_bytes, float fraction,
                   int32_t* evicted, int32_t* n_evicted, ivf_cache_move* moves, int32_t* n_moves);

/*
 * How much to prefetch (App. C "Finding Prefetching Amount"; Sec. 4.1 "Prefetching amount"): the byte
 * budget b_p that minimises t_1 + t_2, where t_1 = t_llm while b_p <= bandwidth * t_llm and
 * b_p / bandwidth beyond it (the copy overlaps the generation that precedes the retrieval) and
 * t_2 = r_miss(b_p) * nprobe * t_cc (the host searches the missed clusters one after the other).
 *   bandwidth   host-to-device bytes per second, > 0        t_llm   seconds of generation, >= 0
 *   nprobe      clusters a search selects, >= 1             t_cc    host seconds per missed cluster, >= 0
 *   budgets, miss_rates   host, n >= 1 measured points of the miss-rate curve: budgets (bytes) strictly
 *               increasing, miss rates in [0, 1] and not rising; the curve is taken as linear between
 *               the points and constant outside them
 *   *amount     out: the best budget in bytes: bandwidth * t_llm (App. C's case 1) unless a measured
 *               point beyond it gives a strictly smaller time (case 2; of equal ones the smallest)
 *   *seconds    out, or NULL: the model's t_1 + t_2 at that budget
 *   *which      out, or NULL: 1 or 2, the case
 * t_1 + t_2 is piecewise linear in b_p, so no other amount can be better.  IVF_EINVAL for arguments
 * outside the stated ranges.  Needs no index and no GPU.  Caller keeps every array.
 */
int ivf_prefetch_amount(double bandwidth, double t_llm, int32_t nprobe, double t_cc,
                        const double* budgets, const double* miss_rates, int32_t n,
                        double* amount, double* seconds, int32_t* which);

/*
 * The host part of the hybrid search on its own (Sec. 4.1 step 3: the clusters of q_out that were
 * not prefetched are searched by CPU threads).  Needs no index and no GPU.
 *   lists     host, cluster-major rows of `dtype`, list c = rows offsets[c] .. offsets[c+1]
 *   offsets   host, enough entries for every listed cluster (c + 1 is read)
 *   ids       host, row -> id, or NULL (id = row)
 *   q         host, d float32         clusters  host, n_clusters lists to scan
 *   out_ids / out_scores   host, room for ivf_host_scan_capacity(k) entries: the candidates the merge step
 *             would receive, unordered, with their float64 scores (inner product, or squared L2)
 *   *n_out    number of candidates written; the k best by (score, id) are among them
 * threads: host threads to use (at least 1).  Caller keeps every array.
 */
int ivf_host_scan(const void* lists, const int64_t* offsets, const int64_t* ids, int32_t d, int dtype,
                  int metric, const float* q, const int32_t* clusters, int32_t n_clusters, int32_t k,
                  int32_t threads, int64_t* out_ids, double* out_scores, int32_t* n_out);
/* Entries ivf_host_scan may write for a search of k results (k' of "Arithmetic" above); 0 when k is
 * outside 1 .. IVF_MAX_K. */
int32_t ivf_host_scan_capacity(int32_t k);

/* Kernel timing with HIP events on compute_stream around each kernel of every search while
 * enabled (adds event records to the stream; leave off when timing throughput).  The kernels are those that a
 * search launches otherwise, too. */
int ivf_profile_enable(ivf_index* index, int on);
int ivf_profile_read(ivf_index* index, ivf_profile* out); /* synchronises compute_stream */
int ivf_profile_reset(ivf_index* index);

/*
 * Cluster cache (Sec. 4.2 "Cache design"; appendix on scheduling and cache: decay-based hotness,
 * cache fraction, eviction and consolidation after each batch).  IVF_PLACE_HOST only.
 *
 * With the cache configured, a cluster copied in by ivf_prefetch is cached with hotness h_init.
 * ivf_cache_end_round closes a round: every cached cluster's hotness becomes h / decay, plus
 * h_inc if a search since the previous round selected the cluster while it was resident; then,
 * while the resident bytes exceed fraction * device_buffer_bytes, the cached cluster of lowest
 * hotness is evicted (equal hotness: the larger cluster index first); the survivors are moved
 * to the front of the device buffer, in their order, so that the freed space is contiguous.
 * The moves run on copy_stream and the call returns when they are enqueued (the next prefetch and
 * the next search are ordered behind them); passing `stats` waits for them, to report their time.
 * Call it between batches, with no ivf_prefetch reset in between that should keep the cache:
 * IVF_PREFETCH_RESET drops the cache too.  Hotness is single precision on the device.
 *   fraction in [0, 1]; h_init >= 0; decay >= 1; h_inc >= 0.  fraction < 0 switches the cache off.
 * ivf_cache_hotness: host array of nlist floats, < 0 for clusters that are not cached.
 */
typedef struct ivf_cache_stats {
    int32_t n_cached;      /* cached clusters when the round ended, before eviction */
    int32_t n_evicted;
    uint64_t bytes_cached; /* their payload bytes, before eviction */
    uint64_t bytes_kept;   /* payload bytes still cached afterwards (= device buffer in use) */
    uint64_t bytes_moved;  /* bytes moved inside the device buffer by the consolidation */
    float ms_update;       /* hotness kernel + read-back */
    float ms_compact;      /* the moves inside the device buffer */
    int32_t n_launches;    /* kernels that carried them out (one per group of moves that do not disturb each other) */
} ivf_cache_stats;
int ivf_cache_configure(ivf_index* index, float fraction, float h_init, float decay, float h_inc);
int ivf_cache_end_round(ivf_index* index, ivf_cache_stats* stats /* or NULL */);
int ivf_cache_hotness(ivf_index* index, float* hotness);

/*
 * Prefetching scheduler (Sec. 4.2 "Scheduling optimization for prefetching"): groups the nq
 * queries of a global batch (host, nq x d float32, nq <= 4096) into micro-batches of `micro`
 * by a greedy search on squared L2 distance, on the GPU.  While queries remain, the remaining
 * query of lowest index seeds a micro-batch and the micro - 1 remaining queries nearest to it
 * follow, nearest first (equal distance: lower index first).  order (host, nq entries) receives
 * the query indices micro-batch after micro-batch; the last micro-batch may be short.
 * *ms_gpu (or NULL) receives the time of the two kernels.  Blocks until order is filled.
 */
int ivf_schedule(ivf_index* index, const float* q, int32_t nq, int32_t micro, int32_t* order, float* ms_gpu);

/*
 * Answering from retrieved passages: the operators of the language model's step behind a retrieval.  The
 * queries of a micro-batch (ivf_schedule) are answered from passages that they share, and the beams of a beam
 * search share their whole prompt, so keys and values lie in a paged cache of which a group of sequences can
 * share a prefix.  These calls need no index.  All pointers are device pointers, work is enqueued on `stream`
 * (a hipStream_t, NULL for the default stream) without waiting, nothing is allocated, and calls may be captured
 * into a graph.  What the arrays on the device hold can change from call to call and from replay to replay.
 *
 * ivf_kv_cache: the keys and values of one layer.  Token slot t is place t % page of page t / page:
 *   element e of head h is at  (t / page) * page_stride + (t % page) * token_stride + h * head_stride + e
 * of k and of v, so pages can hold tokens one after the other or heads one after the other.  Strides count
 * elements and are multiples of 8, those of pages and tokens below 2^30; k and v are 16-byte aligned; dtype is
 * IVF_F16 or IVF_BF16; page is a power of two.
 *
 * ivf_kv_step: the sequences of one step, for all layers.
 *   q_off     [n_seq + 1] first new token of each sequence, ascending from 0 to n_tokens
 *   len       [n_seq] keys that the sequence has of its own, those of its new tokens included: its new tokens
 *             are the last q_off[s + 1] - q_off[s] of them
 *   table     [n_seq][table_stride] entry i names the slots of the sequence's own keys i * page ..: slots
 *             entry * page and on.  `page` here is a power of two of at most the cache's: with page = 1 the table
 *             names every slot by itself, and a beam's past moves by its table row alone (ivf_beam_step)
 *   group_off [n_groups + 1] or NULL (n_groups = 0): sequences group_off[g] .. group_off[g + 1] share the
 *             prefix g of prefix_len[g] keys, in the slots that row g of prefix_table names by entries of
 *             prefix_page slots.  A prefix comes before the own keys.  Sequences outside all groups have none
 *   max_q, max_len, max_prefix  the most new tokens, own keys and prefix keys of any sequence as far as the
 *             caller knows (0: unknown).  They size the launch: lengths beyond them are still computed
 *             right, but slower
 * Key j of a sequence is key j of its prefix, or own key j - prefix_len; new token i has position
 * prefix_len + len - (new tokens) + i.  Of a prefix, and of a sequence's own keys, at most the first 2^30 - 1024
 * count.  Entries outside the cache and lengths outside the tables are not
 * followed out of bounds: such keys are never written, and when read hold what some other slot holds.
 */
typedef struct ivf_kv_cache {
    void* k;
    void* v;
    int64_t n_pages, page_stride, token_stride, head_stride;
    int32_t page, n_heads, d, dtype;
} ivf_kv_cache;

typedef struct ivf_kv_step {
    const int32_t* q_off;
    const int32_t* len;
    const int32_t* table;
    int64_t table_stride;
    const int32_t* group_off;
    const int32_t* prefix_len;
    const int32_t* prefix_table;
    int64_t prefix_stride;
    int32_t n_seq, n_tokens, page, max_q, max_len;
    int32_t n_groups, prefix_page, max_prefix;
} ivf_kv_step;

/* One element vector of d for every head of every token: element e of head h of token t is at
 * t * token_stride + h * head_stride + e.  Strides are multiples of 8, data is 16-byte aligned. */
typedef struct ivf_rows {
    void* data;
    int64_t token_stride, head_stride;
} ivf_rows;

/*
 * Appends the new tokens' keys and values (n_tokens x cache->n_heads x d each, of the cache's type) to the
 * cache, each in the slot of its place, and rotates keys and, with q given, queries by position on the way.
 *   rotary     [n_positions][rot] float32: cosines of the rot / 2 angles of a position, then their sines; or
 *              NULL with rot = 0: nothing is rotated.  rot is a multiple of 16 of at most d; the elements from
 *              rot on are copied.  A pair (a, b) becomes (a c - b s, b c + a s) in 32 bits, rounded once
 *   interleaved  0: pairs are elements (f, f + rot / 2); 1: elements (2 f, 2 f + 1)
 *   positions  [n_tokens] the positions to rotate by (taken into 0 .. n_positions - 1), or NULL: the tokens'
 *              positions in their sequences
 *   q, q_out   n_tokens x n_q_heads x d each, or both NULL with n_q_heads = 0; q_out may be q
 * d is a multiple of 16 of at most 1024.  Tokens whose place is not in the table or whose entry is not in the
 * cache are not written (their queries are rotated).  Two tokens must not share a slot.
 */
int ivf_kv_append(const ivf_kv_step* step, const ivf_kv_cache* cache, const ivf_rows* k, const ivf_rows* v,
                  const float* rotary, int32_t n_positions, int32_t rot, int32_t interleaved, const int32_t* positions,
                  const ivf_rows* q, const ivf_rows* q_out, int32_t n_q_heads, void* stream);

/*
 * Attention of the new tokens over the cache: out = softmax(scale * q . k) v over the keys that a token sees, in
 * 32 bits, rounded once.  A token at position p sees key j when j <= p and, with window > 0, p - j < window or j <
 * sinks.  A token that sees nothing gets zeros.  The keys of a long prefix are read once for all tokens of its group.
 *   q, out     n_tokens x n_q_heads x d, of the cache's type, which do not overlap; query head h reads key
 *              head h / (n_q_heads / cache->n_heads)
 *   lse        [n_tokens][n_q_heads] float32: the logarithm of the sum of the exponentials (-INF: nothing
 *              seen), or NULL
 *   scale      > 0
 *   workspace  device, 16-byte aligned, at least what ivf_attend_workspace() says for the same arguments; its
 *              contents need not be kept, and calls that may overlap need one each
 * d is 64, 96, 128 or 256.  Keys and values in slots that a token does not see never reach its result, whatever
 * they hold; probabilities are rounded to the cache's type before the product with the values.
 */
int ivf_attend_workspace(const ivf_kv_step* step, const ivf_kv_cache* cache, int32_t n_q_heads, int32_t window, int32_t sinks,
                         size_t* bytes);
int ivf_attend(const ivf_kv_step* step, const ivf_kv_cache* cache, const ivf_rows* q, int32_t n_q_heads, const ivf_rows* out,
               float* lse, float scale, int32_t window, int32_t sinks, void* workspace, size_t workspace_bytes, void* stream);

/*
 * One step of a beam search for n_prompts prompts of beams_in beams: of all continuations of a prompt's beams
 * by one token of the vocabulary the beams_out best become the new beams, and rows of per-beam states move.
 * Row r = prompt * beams_in + beam:
 *   logits     row r at r * row_stride (elements of dtype), `vocab` entries; logarithm of the softmax in 32 bits:
 *              (x - max) - log(sum of exp(x - max)).  -INF and NaN entries are no continuations (and count
 *              for nothing in the sum).  Where entries are +INF, these alone are, and share the probability: -log(their number)
 *   scores_in  [rows] the beams' scores; a continuation's score is score + log-softmax.  A beam at -INF
 *              offers nothing
 *   done_in    [rows] or NULL: a beam whose byte is not zero offers only the token `eos`, at its own score
 * Order: larger score, then lower beam, then larger logit, then lower token.
 *   scores_out, parent, token, done_out   [n_prompts][beams_out], best first: the score, the row it continues, the
 *              token, and 1 where the parent was done or the token is eos.  Where a prompt has fewer
 *              continuations: score -INF, parent = its first row, token -1, done 1.  They do not overlap the inputs
 *   states     host array of n_states: row prompt * beams_out + i of `to` becomes row parent of `from`
 *              (row_bytes, and strides in bytes); `to` must not overlap `from`
 *   workspace  as in ivf_attend; its size is ivf_beam_workspace()
 * beams_in and beams_out are at most IVF_MAX_BEAMS, n_states at most IVF_MAX_BEAM_STATES, vocab at most 2^30;
 * logits are IVF_F32, IVF_F16 or IVF_BF16.
 */
#define IVF_MAX_BEAMS 64
#define IVF_MAX_BEAM_STATES 8
typedef struct ivf_beam_state {
    const void* from;
    void* to;
    int64_t row_bytes, from_stride, to_stride;
} ivf_beam_state;
int ivf_beam_workspace(int32_t n_prompts, int32_t beams_in, int32_t vocab, int32_t beams_out, size_t* bytes);
int ivf_beam_step(const void* logits, int64_t row_stride, int dtype, int32_t n_prompts, int32_t beams_in, int32_t vocab,
                  const float* scores_in, const uint8_t* done_in, int32_t eos, int32_t beams_out, float* scores_out,
                  int32_t* parent, int32_t* token, uint8_t* done_out, const ivf_beam_state* states, int32_t n_states,
                  void* workspace, size_t workspace_bytes, void* stream);

/* Number of host threads used for the scan of C_miss (default: hardware threads, at most 64). */
int ivf_set_host_threads(ivf_index* index, int32_t n);

const char* ivf_strerror(int status);
const char* ivf_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* IVF_H */
