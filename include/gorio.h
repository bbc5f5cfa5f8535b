/*
 * gorio.h -- C ABI of the MI355X (gfx950) paged graph beam-search library.
 *
 * The library implements the GPU side of GORIO ("GPU-Centered Remote I/O for
 * Graph ANNS over NVMe-oF"): batched DiskANN-style beam search whose node
 * records live in 4 KB pages.  Every search-side decision is taken on the GPU:
 * how each query advances, which pages it is missing, where a query waiting
 * for pages is kept and when it continues (Sec. 3.1, Fig. 1).  A host proxy
 * thread does nothing but read pages from the backing store and post their
 * completions where the GPU can see them (Sec. 3.3, Sec. 4 "CPU transport
 * proxy").  On one GPU a pinned host-memory backing store with an injected
 * per-request latency takes the place of the remote NVMe-oF namespace of
 * Sec. 4 ("Remote storage").
 *
 * Search semantics (Sec. 1 and Sec. 2.2 describe the search only as a loop
 * that grows a candidate frontier by visiting graph nodes and scoring their
 * neighbours, which in turn names the pages to read next):
 *   key(v) = (squared L2 distance(q, v), v)       -- ties broken by node id
 *   V = {entry};  X = {}
 *   repeat: F = the min(L, |V|) smallest keys of V;
 *           S = the first min(W, .) members of F not in X (in F order);
 *           stop if S is empty;  X += S;
 *           for u in S, for each of u's edges v: if v not in V, V += {v}
 *   result = the first k members of F.
 * Results do not depend on the cache size, the backing latency or the order
 * in which page requests complete.
 *
 * Page layout: node v is stored at slot s = node_to_slot ? node_to_slot[v] : v,
 * position i = s % records_per_page of page s / records_per_page.  Its record
 * is a vector (D x uint8 or D x float32) and an adjacency block ([uint32
 * degree][R x uint32 ids, padded with UINT32_MAX]).  A graph row's UINT32_MAX
 * entries mean "no edge"; the block keeps the row's other ids in order and
 * degree = their count.  Inside a page (bytes not covered below are zero):
 *   vectors first (the default): vector i at byte i * V, where V = vector
 *     bytes rounded up to 16, then adjacency block i at byte
 *     records_per_page * V + i * (record_bytes - V).  For 128-byte vectors
 *     every vector starts on a 128-byte line, so a distance evaluation reads
 *     one line instead of two;
 *   contiguous: record i at byte i * record_bytes, the adjacency block right
 *     after the vector (DiskANN's record order).
 * Both layouts put the same nodes in the same pages; only the bytes inside a
 * page move.
 *
 * Conventions for every call:
 *   - Status codes, never exceptions; gorio_last_error() returns a
 *     thread-local message for the last failing call on this thread.
 *   - The caller owns every array it passes; the library copies what it keeps.
 *   - One thread at a time per index; no call on an index may overlap a
 *     search on it from another thread.  Searches of one index issued on
 *     different streams run one after another: a search on another stream
 *     than the previous search of the index waits on the GPU for that search
 *     (an event the index records), because they share the index's counters;
 *     on the same stream, stream order does it where that stream is the null
 *     or the per-thread stream; on a created stream the search waits for the
 *     event all the same (a stream created after another was destroyed can
 *     get the same handle).  Different indexes may be
 *     used from different threads.
 *   - The device is the HIP device current when gorio_build_index is called;
 *     later calls switch to it and restore the caller's device.
 *
 * Environment (read by each paged search; tuning and test hooks, none needed
 * for normal use):
 *   GORIO_FILL_WAVES       waves that only copy arriving pages (default 32, at most 64)
 *   GORIO_MAX_PENDING      page requests per query, overriding gorio_set_scheduler's
 *   GORIO_HOST_EXECUTOR    host-scheduled lanes: 1 (default) = one persistent launch runs
 *                          the turns the host writes to a ring; 0 = a launch per round
 *   GORIO_TURN_PASSES      host-scheduled lanes: passes that found pages ready before a lane
 *                          yields (default: none with the executor, 2 with a launch per round)
 *   GORIO_FILL_BUDGET_US   launch per round: the fill kernel leaves after this long and is
 *                          launched again (default 2000)
 *   GORIO_ROUND_FLIGHTS    launch per round: round kernels in flight, each on a stream of
 *                          its own (default 2, at most 8)
 *   GORIO_ROUNDS_STATS     1: print the host scheduler's counters to stderr
 *   GORIO_WATCHDOG_S       a paged search still running after this many seconds is
 *                          aborted with GORIO_ETIMEOUT (default 120)
 *   GORIO_PROXY_JITTER_US  extra random delay per page request (completions reorder)
 *   GORIO_PROXY_HOLD       1: the proxy completes nothing (exercises the watchdog)
 *   GORIO_CTRL_STRIDE      spacing of the paged search's control words, in 8-byte words
 *                          (default 32, read when the cache is set)
 */
#ifndef GORIO_H
#define GORIO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gorio_index gorio_index;

typedef enum {
    GORIO_OK = 0,
    GORIO_EINVAL = 1,        /* an argument is out of range or inconsistent */
    GORIO_ENOMEM = 2,        /* device or pinned host allocation failed */
    GORIO_EDEVICE = 3,       /* a HIP runtime call or a kernel failed */
    GORIO_ETIMEOUT = 4,      /* paged search did not finish within the watchdog limit */
    GORIO_EUNSUPPORTED = 5   /* valid request the library does not implement */
} gorio_status;

typedef enum { GORIO_U8 = 0, GORIO_F32 = 1 } gorio_dtype;

/* Arrangement of the bytes inside a page (see the top of this file). */
typedef enum {
    GORIO_LAYOUT_DEFAULT = 0,        /* vectors first */
    GORIO_LAYOUT_VECTORS_FIRST = 1,
    GORIO_LAYOUT_CONTIGUOUS = 2
} gorio_arrangement;

/* Node-record placement in pages.  Zero fields take the default. */
typedef struct {
    uint32_t page_bytes;          /* page size; default 4096; multiple of 16 */
    uint32_t record_bytes;        /* bytes per node; default V + 4 + 4R with V = vec_bytes
                                     (contiguous) or vec_bytes rounded up to 16 (vectors
                                     first); >= that default's minimum, multiple of 4 */
    uint32_t records_per_page;    /* default page_bytes / record_bytes */
    uint32_t arrangement;         /* gorio_arrangement; 0 = default (vectors first) */
    const uint32_t *node_to_slot; /* host array of n entries, a permutation of [0, n); NULL = identity */
} gorio_page_layout;

/* Per-search counters (filled when gorio_search gets a non-NULL stats). */
typedef struct {
    double kernel_ms;          /* GPU time of the search launch(es), HIP events on the search stream */
    double wall_ms;            /* host wall time inside gorio_search */
    uint64_t evaluations;      /* distance evaluations, including re-evaluations */
    uint64_t reevaluations;    /* evaluations whose node could not be recorded in the visited filter
                                  (may repeat an earlier one of the same query) */
    uint64_t expansions;       /* nodes expanded (adjacency lists read) */
    uint64_t iterations;       /* beams expanded, summed over queries */
    uint64_t hits;             /* paged mode: record accesses served by a resident page */
    uint64_t misses;           /* paged mode: record accesses that had to wait for a page */
    uint64_t pages_served;     /* paged mode: pages moved from the backing store into the cache */
    uint64_t bytes_served;     /* paged mode: pages_served * page_bytes */
    uint64_t parks;            /* paged mode: times a query was set aside waiting for pages */
    uint64_t resumes;          /* paged mode: times a parked query was picked up again */
    uint64_t proxy_peak;       /* paged mode: most page requests the proxy held at once */
} gorio_stats;

/* Read-only facts about a built index. */
typedef struct {
    gorio_dtype dtype;
    uint64_t n;
    uint32_t D, R;
    uint32_t page_bytes, record_bytes, records_per_page;
    int vectors_first;         /* 1: vectors-first pages, 0: contiguous records */
    uint64_t num_pages;
    uint64_t index_bytes;      /* num_pages * page_bytes */
    uint32_t entry;            /* entry node used by every search */
    int resident;              /* 1: all pages in HBM; 0: paged through the HBM cache */
    uint64_t cache_slots;      /* paged mode: number of page slots in the HBM cache */
    int device;                /* HIP device ordinal */
} gorio_index_info;

/*
 * Build an index: pack records into pages and choose the entry node.  The
 * index is a DiskANN-style graph (Sec. 5.1) stored as fixed-size graph pages
 * that are the unit of every read (Sec. 3.1, Fig. 1: graph pages on the remote
 * namespace; Sec. 4 "Remote storage": the page-cache path fetches whole
 * pages).  Record and page layout as described at the top of this file.
 *   vectors: host, n x D row-major (uint8 or float32 per dtype).
 *   graph:   host, n x R row-major uint32; UINT32_MAX = no edge; any other id must be < n.
 *   layout:  NULL = all defaults.
 *   entry:   UINT32_MAX = medoid rule: the node nearest (squared L2, ties to the
 *            smaller id) to the centroid c, where for uint8 c_d = floor((sum_i x_id
 *            + floor(n/2)) / n) and for float32 c_d = (float)(sum_i (double)x_id / n)
 *            summed in i order; otherwise the given node (< n).
 * Limits: 1 <= n < 2^31; uint8: D % 4 == 0, D <= 512; float32: D <= 256; 1 <= R <= 256.
 * The packed index is placed in HBM (resident mode).  *out is set only on GORIO_OK.
 */
gorio_status gorio_build_index(gorio_dtype dtype, const void *vectors, uint64_t n, uint32_t D,
                               const uint32_t *graph, uint32_t R,
                               const gorio_page_layout *layout, uint32_t entry,
                               gorio_index **out);

/*
 * Size the HBM page cache (GORIO Sec. 3.2: GPU page cache with a per-slot ready
 * table; Sec. 4: BaM-derived page-cache path).
 * bytes >= index_bytes: resident mode, every page in HBM, no misses.
 * otherwise: paged mode with floor(bytes / page_bytes) slots; the pages move
 * to a pinned host backing store and the cache starts cold.  Too few slots for
 * the configured query slots to make progress -> GORIO_EINVAL.
 */
gorio_status gorio_set_cache(gorio_index *ix, uint64_t bytes);

/*
 * Configure the backing-store proxy for paged mode (Sec. 3.3 / Sec. 4: the
 * proxy batches submissions and completions and caps outstanding remote I/O).
 *   latency_us:      injected delay from a page request's publication to its completion (>= 0).
 *   max_outstanding: cap on requests the proxy holds in flight (0 = default 4096).
 *   oversub:         query slots per resident wavefront of the persistent kernel (1..16).
 *   blocking:        scheduling mode.
 *                    0 = split-phase: the persistent GPU scheduler parks a query
 *                        on a missing page and runs other ready queries (Sec. 3.3);
 *                    1 = wait in place for each missing page, one query per wave
 *                        (the blocking demand-paging path the paper compares
 *                        against, Sec. 5.1, Table 2);
 *                    2 = host-scheduled lanes: a host thread (the caller's)
 *                        keeps the query lanes and decides which runs next, as
 *                        their pages are filled; a persistent GPU launch runs the
 *                        turns it hands over through a ring in host memory (or,
 *                        with GORIO_HOST_EXECUTOR=0, a launch per round), using
 *                        the same page cache, descriptors and proxy (the
 *                        GustANN-style scheduler over GORIO's backend that the
 *                        paper compares against, Sec. 5.1, Table 2).  oversub is
 *                        ignored; the lanes are min(query_waves or 8 per compute
 *                        unit, slots / (2 * max_pending), nq, 8192).
 *                    3 = GPU resume queue (Sec. 3.1, Fig. 1: a ready table
 *                        feeding a resume queue): the same lanes, with their
 *                        state in HBM, but nothing on the host except the proxy
 *                        and the watchdog; a lane that parks joins the waiter
 *                        set of each cache slot it waits for, the fill wave
 *                        that makes a slot READY queues those lanes in a run
 *                        queue in HBM, and executor waves of one persistent
 *                        launch run the queued lanes' turns.  oversub is
 *                        ignored; the lanes are counted as in mode 2.
 *                    Results are the same in every mode.
 * Takes effect at the next search.  Ignored in resident mode.
 * Errors: GORIO_EINVAL for a NULL index or an argument out of range.
 */
gorio_status gorio_set_backing(gorio_index *ix, double latency_us, uint32_t max_outstanding,
                               uint32_t oversub, int blocking);

/*
 * Shape of the paged scheduler (Sec. 3.3: the persistent scheduler runs many
 * queries per wave and caps the page requests in flight).
 *   query_waves: most waves that run queries (0 = 8 per compute unit).
 *   max_pending: page requests one query keeps outstanding (1..256; 0 = 32).
 * A search runs min(query_waves * oversub, slots / (2 * max_pending), nq)
 * queries at once, in ceil(that / oversub) waves (one query per wave when
 * blocking): every query may pin max_pending slots, and half of the cache is
 * kept free for the clock to evict.  With equal query_waves, the blocking
 * mode therefore holds oversub times fewer queries than the split-phase mode,
 * which is the comparison of Sec. 5.2 (waits in place vs. yields and runs
 * other queries).  Takes effect at the next search; ignored in resident mode.
 * Errors: GORIO_EINVAL for a NULL index, query_waves > 65536 or
 * max_pending > 256.
 */
gorio_status gorio_set_scheduler(gorio_index *ix, uint32_t query_waves, uint32_t max_pending);

/*
 * Batched search (GORIO Sec. 3.3: persistent scheduler; each query is finished
 * or parked on a missing page and later resumed).
 *   queries: nq x D (uint8 or float32), host or device pointer.
 *   ids:     nq x k uint32 out; dists: nq x k out, int32 (uint8 data) or float32.
 *            Both host or device pointers (detected per pointer).  Host
 *            buffers are staged through a device buffer the index keeps
 *            (grown when a batch needs more) and the call returns once the
 *            answers are back in them.
 *   Slots past the reachable set are padded with UINT32_MAX and INT32_MAX / +inf.
 *   stats:   NULL or a struct to fill; non-NULL makes the call wait for the search.
 *   stream:  hipStream_t to launch on (NULL = the null stream).  With device
 *            pointers and stats == NULL a resident search returns without
 *            waiting; a paged search always returns when it is done (the
 *            calling thread runs its watchdog, and in mode 2 its scheduler).
 * Requires 1 <= k <= L <= 256 and 1 <= W <= L (paged: W <= 64).  nq == 0 is a
 * no-op.  Errors: GORIO_EINVAL for arguments out of range, GORIO_EUNSUPPORTED
 * for a paged W above 64, GORIO_ENOMEM / GORIO_EDEVICE from the device,
 * GORIO_ETIMEOUT when a paged search did not finish within the watchdog
 * limit (the counters so far are filled; the cache is reset), and
 * GORIO_EUNSUPPORTED on a stream under graph capture (each search takes its
 * query tickets from a base the host advances, so a replay would be wrong;
 * gorio_search_noalloc is the entry point to capture).
 */
gorio_status gorio_search(gorio_index *ix, const void *queries, uint64_t nq,
                          uint32_t k, uint32_t L, uint32_t W,
                          uint32_t *ids, void *dists, gorio_stats *stats, void *stream);

/*
 * gorio_search for callers that cannot allocate memory: code running under
 * HIP graph capture, serving loops and harnesses that forbid hipMalloc.  It
 * allocates nothing and stages nothing; the caller passes device buffers.
 * Resident indexes only (a paged index -> GORIO_EUNSUPPORTED).
 *   queries, ids, dists: device pointers, as for gorio_search (host pointers
 *            -> GORIO_EINVAL).  k, L, W and nq: as for gorio_search.
 *   stats:   NULL, or filled with kernel_ms, evaluations, reevaluations,
 *            expansions and iterations (the call then waits for the search).
 *   stream:  hipStream_t (NULL = the null stream).
 * Under graph capture on `stream` the call records and waits for no event
 * (the caller orders the graph's replays with other work on the index) and
 * takes no statistics (stats != NULL -> GORIO_EINVAL); every replay clears
 * the scratch and runs the whole search again.
 * Scratch: the search's counters live in a fixed 128-byte device array of
 * the library, one per GPU, kept until the process ends; no batch size needs
 * more.  Each call clears it first.  Calls that overlap on one GPU (different
 * indexes, streams or threads) share that array and race; serialise them.
 * Results are the same as gorio_search's.
 */
gorio_status gorio_search_noalloc(gorio_index *ix, const void *queries, uint64_t nq,
                                  uint32_t k, uint32_t L, uint32_t W,
                                  uint32_t *ids, void *dists, gorio_stats *stats, void *stream);

/* Facts about the index (entry node, page counts, mode). */
gorio_status gorio_index_info_get(const gorio_index *ix, gorio_index_info *info);

/*
 * Copy `count` packed pages starting at page `first` to host memory `dst`
 * (count * page_bytes bytes), from HBM or the backing store.
 */
gorio_status gorio_copy_pages(const gorio_index *ix, uint64_t first, uint64_t count, void *dst);

/*
 * Locality-aware node placement (host only; no device is touched): fills
 * node_to_slot (n entries, a permutation of [0, n)) so that graph neighbours
 * share pages, for use as gorio_page_layout.node_to_slot.  Graph pages are the
 * unit of I/O (Sec. 3.1); the disk-resident ANNS work the paper builds on
 * places neighbours together for this reason (Sec. 6).  Rule: visit nodes
 * breadth-first from `entry`, neighbours in adjacency order; a visited node
 * without a slot takes the next slot and then fills the rest of its page
 * (records_per_page slots) with its own slot-less neighbours, in adjacency
 * order; unreached nodes follow in id order.  Deterministic.
 *   graph: host, n x R row-major; UINT32_MAX = no edge; other ids must be < n.
 * Errors: GORIO_EINVAL for NULL pointers, n, R or records_per_page out of range,
 * entry >= n or a bad id.
 */
gorio_status gorio_locality_order(const uint32_t *graph, uint64_t n, uint32_t R, uint32_t entry,
                                  uint32_t records_per_page, uint32_t *node_to_slot);

/*
 * Cluster placement (host call; runs on the current HIP device): k-means on
 * the vectors, then node_to_slot places the nodes cluster by cluster (id order
 * inside a cluster), for use as gorio_page_layout.node_to_slot.  Graph pages
 * are the unit of I/O (Sec. 3.1) and page layout and graph locality decide how
 * much of a fetched page a search uses (Sec. 6, DiskANN and Starling); a paged
 * cache holds a few clusters' pages at once, so placing nodes by cluster and
 * admitting queries by cluster (gorio_set_query_order) lets queries in flight
 * reuse each other's pages.
 *   vectors:    host, n x D row-major, uint8 or float32 per dtype.
 *   clusters:   K centroids, 1 <= K <= min(n, 65536).  Initial centroids are the
 *               vectors of nodes floor(i n / K); then `iterations` (<= 64) Lloyd
 *               steps (nearest centroid by squared L2 in float32 on the GPU, ties to
 *               the smaller index; each centroid becomes the mean of its members,
 *               an empty one stays).
 *   node_to_slot: host out, n entries, a permutation of [0, n).
 *   centroids:  host out, K x D float32 (the final centroids).
 * Deterministic.  Results of a search never depend on the placement.
 * Device memory during the call: the vectors, 20 bytes per node, at most 256 MB
 * of counts, about 12 K D bytes of centroids and, with iterations, 8 K D (uint8)
 * or 128 K D (float32) bytes of sums.
 * Errors: GORIO_EINVAL for NULL pointers or n, D (1..1024), K, iterations out of
 * range; GORIO_ENOMEM / GORIO_EDEVICE from the device.
 */
gorio_status gorio_cluster_order(gorio_dtype dtype, const void *vectors, uint64_t n, uint32_t D,
                                 uint32_t clusters, uint32_t iterations, uint32_t *node_to_slot,
                                 float *centroids);

/*
 * Admission order of paged searches (the persistent scheduler of Sec. 3.3
 * decides which query a free slot takes next): with K > 0 centroids each paged
 * search first assigns every query to its nearest centroid (squared L2 in
 * float32, ties to the smaller index) and admits the queries cluster by
 * cluster, in index order inside a cluster, so the queries in flight share
 * pages (the cross-query reuse that Sec. 7.2 names as miss coalescing).  Each
 * query's answer is unchanged and is written to its own row.  Resident
 * searches ignore the order.
 *   centroids: host, K x D float32 (e.g. from gorio_cluster_order); copied.
 *   clusters:  K, 0 <= K <= 65536; 0 restores index order.
 * Errors: GORIO_EINVAL for a NULL index, K > 65536, or NULL centroids with K > 0.
 */
gorio_status gorio_set_query_order(gorio_index *ix, const float *centroids, uint32_t clusters);

/*
 * Release everything the index owns: its HBM pages or cache, the ready-table
 * words and rings of Sec. 3.2, the pinned backing store and the proxy thread
 * of Sec. 3.3 / Sec. 4 ("CPU transport proxy"), which is stopped first.  Must
 * not overlap a search on the index.  NULL is a no-op.
 */
void gorio_free_index(gorio_index *ix);

/* ---------------------------------------------------------------------------
 * Keys and values of passages, in pages.
 *
 * What a search finds is read next: a program that answers from the nodes
 * found keeps the attention keys and values of each node's text in pages in
 * HBM, beside the index, and runs its model's new tokens over the pages of the
 * nodes that the search returned.  These calls do that, once a step (attach,
 * plan, share) and once a layer (store, attend):
 *
 *   gorio_kv_attach  a search's ids -> each request's table of pages
 *   gorio_kv_plan    request lengths -> starts, positions and slots of the new
 *                    tokens, and the tables grown by pages of a free list
 *   gorio_kv_store   the new tokens' keys and values -> their slots
 *   gorio_kv_attend  attention of the new tokens over the pages
 *   gorio_kv_load    rows of the pages at given slots
 *   gorio_kv_share, gorio_kv_attend_shared  for batches in which neighbouring
 *                    requests' tables begin with the same pages
 *
 * A request's tokens have virtual positions 0, 1, ...; position j is place
 * j % page_tokens of the page that entry j / page_tokens of the request's row
 * of the table names.  An entry outside [0, num_pages) names no page.
 * A token's slot is page * page_tokens + place.
 *
 * Conventions, besides those above: every array is in device memory (of one
 * GPU, which the call switches to); the calls allocate nothing, wait for
 * nothing and only enqueue kernels on `stream`, so they can be captured into
 * a HIP graph.  A size of zero (no request, no token) is a no-op.  Lengths are
 * read on the GPU: a value there that makes no sense (negative, past a
 * capacity) is clamped as each call says and never reaches memory outside the
 * arrays.  Errors: GORIO_EINVAL (NULL or host pointers, sizes out of range,
 * misaligned pointers or strides), GORIO_EUNSUPPORTED (a combination of types
 * that there is no kernel for), GORIO_EDEVICE.
 * ------------------------------------------------------------------------- */

typedef enum { GORIO_KV_BF16 = 0, GORIO_KV_F16 = 1, GORIO_KV_E4M3 = 2, GORIO_KV_MX8 = 4, GORIO_KV_MX4 = 5 } gorio_kv_dtype;

/* GORIO_KV_MX8 and GORIO_KV_MX4 are the microscaling formats of the Open Compute
 * Project with e4m3 and e2m1 elements: elements 32 i .. 32 i + 31 of a row share
 * a power of two, 2^E, kept as the byte E + 127.  An element stands for its
 * value times 2^E; where the byte is 255, the elements stand for NaN.  e2m1 has
 * the values 0, 0.5, 1, 1.5, 2, 3, 4 and 6 (codes 0..7) and their negatives
 * (8..15), two a byte, the element with the even index in the low half. */

/* The pages of one layer.  Element d of head h's key at place i of page p is
 * keys[p * page_stride + h * head_stride + i * token_stride + d]; values alike. */
typedef struct {
    uint32_t dtype;         /* gorio_kv_dtype of keys and values */
    uint32_t heads;         /* key and value heads, 1..1024 */
    uint32_t D;             /* elements of a head: a multiple of 8, 8..256; of 32 with GORIO_KV_MX8, _MX4 */
    uint32_t page_tokens;   /* 1..65536 */
    uint64_t num_pages;     /* 1..2^31 - 1 */
    void *keys, *values;    /* 16-byte aligned */
    uint64_t page_stride, head_stride, token_stride;  /* elements, multiples of 8 (of 32 with
                               GORIO_KV_MX8, _MX4); all three 0 = packed pages, [page][head][token][D] */
    const float *key_scale, *value_scale;  /* GORIO_KV_E4M3: `heads` factors each; an element
                               stands for its 8-bit value times its head's factor.  NULL = 1 */
    uint8_t *key_powers, *value_powers;  /* GORIO_KV_MX8, _MX4: the powers' bytes, at the 32nd part
                               of their elements' offset: block i of the key above is
                               key_powers[(p * page_stride + h * head_stride + place * token_stride) / 32 + i].
                               Not read with other types */
} gorio_kv_cache;

/* One call's new tokens, and what they see. */
typedef struct {
    uint32_t dtype;         /* gorio_kv_dtype of q and out: GORIO_KV_BF16 or GORIO_KV_F16, and that
                               of the pages unless these hold 8 or 4 bits */
    uint32_t heads;         /* query heads, a multiple of the cache's; head h reads head
                               h / (heads / cache heads) */
    uint32_t requests, width;  /* rows and columns of tables */
    uint64_t tokens;        /* rows of q and out */
    const void *q;          /* token t's head h at q + t * q_stride + h * D, 16-byte aligned */
    void *out;              /* laid out alike, with out_stride */
    uint64_t q_stride, out_stride;  /* elements, multiples of 8; 0 = heads * D */
    float *lse;             /* tokens x heads out, or NULL: log of the sum of exp(score) */
    const int32_t *starts;  /* requests + 1: request b's new tokens are rows starts[b]..starts[b+1] */
    const int32_t *lens;    /* requests: all of its tokens, the new ones last */
    const int32_t *tables;  /* requests x width pages */
    const int32_t *fills;   /* requests x width: tokens that a page holds, from its first place
                               (NULL: page_tokens) */
    const int32_t *prefix;  /* requests: its first positions, which every new token sees (NULL: 0) */
    const float *slopes;    /* heads: see below (NULL: 0) */
    float scale, cap;       /* cap 0 = none; cap and |scale| at most 1e38 */
    uint32_t window;        /* 0 = none */
    uint32_t max_new;       /* the most new tokens of a request, if the caller knows it (0: not);
                               chooses a kernel, and changes no result beyond rounding */
} gorio_kv_attention;

/*
 * A search's answers -> tables of pages.  Passage (node) v has tokens[v]
 * tokens in ceil(tokens[v] / page_tokens) pages from first_page[v] on.  Row b
 * of the table gets the pages of nodes[b][0], nodes[b][1], ... one passage
 * after the other, each from a page's first place, as long as whole passages
 * fit into `limit` entries: the first that does not fit ends the row.  Ids at
 * or past n (a search's padding) and passages that have no pages, whose first
 * page is negative, are passed over.
 *   nodes:    requests x k (1 <= k <= 1024), e.g. from gorio_search.
 *   tables, fills: requests x width out: pages and the tokens that each holds;
 *             entries past the passages get -1 and page_tokens.
 *   lens:     requests out: page_tokens times the entries taken, which is the
 *             next position (a passage's last page is never written to by a
 *             request), and the prefix for gorio_kv_attend.
 *   attached: requests out, or NULL: passages in the row.
 * No array that is written overlaps another.
 */
gorio_status gorio_kv_attach(const uint32_t *nodes, uint64_t requests, uint32_t k,
                             const int32_t *first_page, const int32_t *tokens, uint64_t n,
                             uint32_t page_tokens, uint32_t width, uint32_t limit,
                             int32_t *tables, int32_t *fills, int32_t *lens, int32_t *attached,
                             void *stream);

/*
 * A step's plan from request lengths: request b has before[b] tokens and
 * takes added[b] new ones (negative values count as 0).
 *   free_pages: n_free pages that no request holds; request by request, in
 *             order, each takes as many as its entries need from the front.
 *   tables:   requests x width, in and out: the new entries are written.  An
 *             entry for which no page is left gets -1; entries at or past
 *             width are not kept, and take no page.
 *   lens:     requests out: before + added.
 *   starts:   requests + 1 out: exclusive sums of added.
 *   positions, slots: `tokens` out: each new token's position and slot (-1
 *             where it has no page; -1 both past the last new token; new
 *             tokens past `tokens` are left out).
 *   taken:    1 out: pages that the entries needed, which may pass n_free.
 * positions, slots and taken may be NULL.  lens and before are different arrays;
 * no array that is written overlaps another.
 */
gorio_status gorio_kv_plan(const int32_t *before, const int32_t *added, uint64_t requests,
                           uint32_t page_tokens, const int32_t *free_pages, uint64_t n_free,
                           int32_t *tables, uint32_t width, uint64_t tokens, int32_t *lens,
                           int32_t *starts, int32_t *positions, int64_t *slots, int32_t *taken,
                           void *stream);

/*
 * Keys and values of new tokens -> their slots.  Token t's head h is at
 * keys + t * key_stride + h * D (elements, multiples of 8; 0 = heads * D; 16-byte
 * aligned), values alike.  A slot outside the pages stores nothing; slots of
 * one call are distinct.  Into GORIO_KV_E4M3 pages an element is divided by its
 * head's factor, clamped to +-448 and rounded to the nearest (ties to even).
 * Into GORIO_KV_MX8 (MX4) pages: with a the largest size among a block's 32
 * elements, E is the smallest number in -127..127 with a <= 448 * 2^E (6 * 2^E),
 * so that no element is clamped, and each is divided by 2^E and rounded to the
 * nearest (ties to even).  A block that holds a NaN or an infinity gets the byte
 * 255 and elements of 0: all of it stands for NaN.
 *   dtype: of keys and values: the pages' type, or either 16-bit type for
 *          pages of 8 or 4 bits.
 */
gorio_status gorio_kv_store(const gorio_kv_cache *cache, gorio_kv_dtype dtype, const void *keys,
                            const void *values, uint64_t tokens, uint64_t key_stride,
                            uint64_t value_stride, const int64_t *slots, void *stream);

/*
 * Rows of the pages at `tokens` slots -> keys and values, laid out as those of
 * gorio_kv_store (for other pages, for checks, for keys that are turned to
 * other positions).  An element is what it stands for, rounded to the nearest
 * of the rows' type (past its range to an infinity); a slot outside the pages
 * gives a row of zeros, and a slot may be named more than once.
 *   dtype: of keys and values: the pages' type, or either 16-bit type for
 *          pages of 8 or 4 bits.
 * Neither array shares memory with the other or with the cache.
 */
gorio_status gorio_kv_load(const gorio_kv_cache *cache, gorio_kv_dtype dtype, const int64_t *slots,
                           uint64_t tokens, void *keys, void *values, uint64_t key_stride,
                           uint64_t value_stride, void *stream);

/*
 * Which requests of a batch have their first pages in common (a prompt, or
 * passages, that they were all given), for gorio_kv_attend_shared.  Requests
 * b - 1 and b share common[b] positions: page_tokens times the number of leading
 * entries in which their rows of the table, and of fills, are equal, but no
 * more than the whole pages of held[b - 1] and of held[b].  Request b joins the
 * group of the request before it if common[b] >= max(least, 1); the others
 * begin a group each.  Order the requests so that those with the same pages
 * follow one another.
 *   tables:   requests x width; fills (or NULL) alike.
 *   held:     requests: positions that all of a request's new tokens see, as far
 *             as a window lets them: its tokens before the step, or its prefix.
 *   least:    fewer positions than this are not worth a group's own work.
 *   common:   requests out; common[0] = 0.
 *   first:    requests + 1 out: group g is requests first[g]..first[g+1]; entries
 *             past the last group hold `requests`, which makes empty groups.
 *   shared:   requests out: what a request shares with all of its group, the
 *             smallest of their common (0 for a request alone).
 * requests is at most 2^20.  No array that is written overlaps another.
 */
gorio_status gorio_kv_share(const int32_t *tables, const int32_t *fills, const int32_t *held,
                            uint64_t requests, uint32_t width, uint32_t page_tokens, uint32_t least,
                            int32_t *common, int32_t *first, int32_t *shared, void *stream);

/*
 * Attention of new tokens over pages.  New token i of request b stands at
 * position p = lens[b] - (starts[b+1] - starts[b]) + i; its keys and values
 * are read from the pages like all others (store them first).  Key j is
 * visible to it if its table entry names a page, j % page_tokens is below the
 * page's fill, j < lens[b], and (j <= p and p - j < window, or j < prefix[b]).
 *   s_j = scale * (q . k_j); with a cap, s_j = cap * tanh(s_j / cap); then
 *   s_j -= slopes[h] * |p - j|   (a capped score is good to 2^-15 up to a cap of 64, and to
 *                                 2^-20 of itself past that)
 *   out = sum_j exp(s_j) v_j / sum_j exp(s_j) over the visible keys
 * Sums and the softmax are held in 32 bits, its weights rounded to q's type
 * for the product with the values.  A row that sees no key (or whose scores
 * are all -inf) gives zeros and an lse of -inf.  Keys and values that a row
 * does not see do not reach it, whatever they hold.  Elements of GORIO_KV_MX8 and _MX4 pages are
 * read as the nearest values of q's type.  Rows of q past starts[requests] are left
 * as they are in out.  starts is clamped to [0, tokens] and has to ascend.
 *   workspace: gorio_kv_workspace bytes of device memory, 16-byte aligned, for
 *              this call alone until it has run (NULL if 0).  Rows of few new
 *              tokens over long texts are computed in parts, which it holds.
 */
gorio_status gorio_kv_attend(const gorio_kv_cache *cache, const gorio_kv_attention *a,
                             void *workspace, uint64_t workspace_bytes, void *stream);

/* Bytes of workspace that gorio_kv_attend needs; from the sizes alone, no pointer is read. */
gorio_status gorio_kv_workspace(const gorio_kv_cache *cache, const gorio_kv_attention *a,
                                uint64_t *bytes);

/* Groups of neighbouring requests that have their first pages in common, as gorio_kv_share finds
 * them.  Every request is in one of them. */
typedef struct {
    uint32_t groups;        /* 1..requests; some may be empty */
    const int32_t *first;   /* groups + 1: group g is requests first[g]..first[g+1]; ascends from 0 to requests */
    const int32_t *shared;  /* requests: positions that a request shares with its group, the same for
                               all of a group */
} gorio_kv_sharing;

/*
 * gorio_kv_attend for a batch in which requests share a long prefix: the keys
 * and values of the positions below shared[b] are read once for all rows of b's
 * group, and not once for each request.  As far as that goes, a group's rows of
 * tables (and fills) are alike, as gorio_kv_share finds them: a position is
 * looked up in the row of the group's first request or in the request's own.
 * The result is that of gorio_kv_attend beyond rounding, whatever else the call
 * asks for: what a row sees of the shared positions goes by its own position,
 * prefix, window and length.  Groups take launches of their own: up to 12 us
 * where nothing is shared, 20 to 40 where little is.  A call with a window and
 * without a prefix, or whose tables have little room, is computed as by
 * gorio_kv_attend.
 *   workspace: gorio_kv_workspace_shared bytes, about tokens * heads * (D + 2)
 *              floats more than without (545 MB for 32768 tokens of 32 heads of
 *              128): the sums over the shared positions.
 */
gorio_status gorio_kv_attend_shared(const gorio_kv_cache *cache, const gorio_kv_attention *a,
                                    const gorio_kv_sharing *sharing, void *workspace,
                                    uint64_t workspace_bytes, void *stream);

/* Bytes of workspace that gorio_kv_attend_shared needs: from the sizes, and with a window from
 * whether prefix is NULL; no pointer is read. */
gorio_status gorio_kv_workspace_shared(const gorio_kv_cache *cache, const gorio_kv_attention *a,
                                       const gorio_kv_sharing *sharing, uint64_t *bytes);

/*
 * Message for the last failing call on this thread ("" if none).  Errors are
 * returned as status codes so that no failure of the transport path (Sec. 4)
 * or of a search crosses the ABI as an exception; the text says which check
 * or which HIP call failed.  The pointer stays valid until the next failing
 * call on the same thread.
 */
const char *gorio_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* GORIO_H */
