/*
 * wave.h -- C ABI of the wave-index library for AMD MI355X (gfx950).
 *
 * The library implements the data-parallel hot path of the wave index of
 * "RetroInfer: A Vector Storage Engine for Scalable Long-Context LLM
 * Inference": the segmented spherical k-means that builds the cluster index
 * over a key/value cache (section "Wave Index", paragraphs "Index
 * Organization" and "Lightweight Index Construction and Updates") and the
 * decode step that replaces full attention by tripartite attention (paragraph
 * "Tripartite Attention Approximation", the estimation equations, and the
 * decode steps 1-4 of the system overview).
 *
 * Conventions
 *  - Every pointer marked DEVICE is caller-owned GPU memory; HOST pointers are
 *    ordinary host memory.  The library allocates no device memory and keeps
 *    no state between calls (the optional profiler below excepted).
 *  - Every call returns a wave_status; nothing aborts or throws.  Argument
 *    errors are found on the host before any kernel is launched.
 *  - wave_index_build and wave_attention_decode only ENQUEUE work on the given
 *    HIP stream (a hipStream_t passed as void*; NULL is the default stream).
 *    Results are valid once the caller has synchronised that stream.  Two
 *    calls that share a workspace must be ordered on one stream.
 *  - Tensors are dense, row-major, last index fastest.  dtype is the storage
 *    type of q, K, V and of the index's floating arrays.  Accumulation is
 *    fp32 in decode and fp64/fp32-MFMA in the build (see each call).
 *  - Notation follows the paper: d head dimension, N context tokens, p steady
 *    tokens (n_sink + n_local), m clusters per (sequence, KV head), r retrieved
 *    clusters, C centroids, s sizes, VS value sums, L segment length, k
 *    clusters per segment, T k-means iterations, G = Hq / Hkv.
 *  - Supported shapes: d in {64, 128}; 1 <= G <= 8; dtype f32 or bf16;
 *    clusters_per_segment <= WAVE_MAX_CLUSTERS_PER_SEGMENT (8192: one segment
 *    over a 128K-token sequence at 16 tokens per cluster, the "global k-means"
 *    of the segment-size study); N < 2^31.
 */
#ifndef WAVE_H
#define WAVE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  WAVE_OK = 0,
  WAVE_ERR_ARG = 1,             /* null pointer, negative count, iters < 1, ...        */
  WAVE_ERR_SHAPE = 2,           /* unsupported d, G, k, or inconsistent dimensions     */
  WAVE_ERR_DTYPE = 3,           /* dtype not WAVE_F32 / WAVE_BF16                      */
  WAVE_ERR_WORKSPACE = 4,       /* workspace null, misaligned (256 B) or too small     */
  WAVE_ERR_STEADY_MISMATCH = 5, /* decode's n_sink/n_local differ from the index's     */
  WAVE_ERR_HIP = 6              /* a HIP runtime call or kernel launch failed          */
} wave_status;

typedef enum { WAVE_F32 = 0, WAVE_BF16 = 1 } wave_dtype;

enum { WAVE_MAX_CLUSTERS_PER_SEGMENT = 8192 };

/* Index of B x Hkv independent (sequence, KV head) units: the meta index
 * (centroid, value sum, size per cluster: "Index Organization" and the value-sum
 * equation) and the cluster-contiguous key/value rows.  Plain data; the caller
 * fills the dimension fields, calls wave_index_plan for S, m, N_idx and the
 * buffer sizes, allocates the nine buffers on the DEVICE and stores the
 * pointers.  Copying the arrays copies the index. */
typedef struct {
  int32_t dtype;                /* wave_dtype                                          */
  int32_t B, Hkv, d, N;
  int32_t n_sink, n_local;      /* steady zone: first n_sink and last n_local tokens,  */
                                /* attended by position and excluded from clustering   */
  int32_t segment_len;          /* L                                                   */
  int32_t clusters_per_segment; /* k; a ragged last segment of L_s tokens has          */
                                /* min(k, L_s) clusters                                */
  int32_t S, m, N_idx;          /* derived: segments, clusters and indexed tokens per  */
                                /* unit; N_idx = N - (steady tokens)                   */
  int32_t p;                    /* derived: steady tokens = min(N, n_sink) + local part */
  int32_t steady_capacity;      /* rows allocated per unit in k_steady and v_steady: 0  */
                                /* means p (dense); see row_capacity                    */
  void *centroids;              /* DEVICE [B,Hkv,m,d] dtype: mean of raw member keys   */
  void *vsum;                   /* DEVICE [B,Hkv,m,d] dtype: sum of member values      */
  int32_t *sizes;               /* DEVICE [B,Hkv,m]     0 = empty cluster              */
  int32_t *offsets;             /* DEVICE [B,Hkv,m+1]   rows of cluster c in k_perm /  */
                                /*        v_perm are [offsets[c], offsets[c+1])        */
                                /*        (with cluster_capacity > 0 these four have   */
                                /*        cluster_capacity (+ 1) entries per unit)     */
  int32_t *perm;                /* DEVICE [B,Hkv,N_idx] original position of each row  */
  void *k_perm, *v_perm;        /* DEVICE [B,Hkv,N_idx,d] dtype, rows ordered by       */
                                /*        (segment, cluster, original position); with  */
                                /*        row_capacity > 0 the three have row_capacity */
                                /*        rows per unit, the first N_idx in use        */
  void *k_steady, *v_steady;    /* DEVICE [B,Hkv,p,d] dtype: sink rows then local rows */
                                /*        (steady_capacity rows per unit if that is set) */
  int32_t appended_segments;    /* update segments appended by wave_index_append (0 for */
                                /* a freshly built index); they follow the S - this     */
                                /* many segments of the build                           */
  int32_t update_segment_len;   /* their length U and ...                               */
  int32_t update_clusters;      /* ... clusters per update segment (min(k_u, U) each)   */
  int32_t row_capacity;         /* rows allocated per unit in perm, k_perm and v_perm:   */
                                /* 0 means N_idx (dense); a larger value, set by the    */
                                /* caller before wave_index_plan, leaves room for       */
                                /* wave_index_append to add rows in place               */
  int32_t cluster_capacity;     /* clusters allocated per unit in centroids, vsum, sizes */
                                /* (and + 1 entries in offsets): 0 means m (dense); a    */
                                /* larger value, set by the caller before                */
                                /* wave_index_plan, leaves room for wave_index_append to */
                                /* add clusters in place; the first m (m + 1) entries of */
                                /* a unit are in use                                     */
} wave_index;

enum { WAVE_INDEX_BUFFERS = 9 };

/* Host only.  Reads the dimension fields of *ix, writes S, m, N_idx, p into it
 * and the byte size of each of the nine buffers into bytes[] in the order
 * centroids, vsum, sizes, offsets, perm, k_perm, v_perm, k_steady, v_steady.
 * build_workspace_bytes (may be NULL) receives the scratch wave_index_build
 * needs; decode_workspace_bytes (may be NULL) the scratch wave_attention_decode
 * needs for Hq query heads and topk_clusters retrieved clusters.  Sizes of
 * zero-length buffers are reported as 0; their pointers may be NULL. */
wave_status wave_index_plan(wave_index *ix, size_t bytes[WAVE_INDEX_BUFFERS],
                            size_t *build_workspace_bytes, int Hq, int topk_clusters,
                            size_t *decode_workspace_bytes);

/* Index update during decoding ("Lightweight Index Construction", last
 * paragraph): n_new new tokens per unit join the local window of the steady
 * zone; whenever the window holds a whole update segment of U tokens beyond
 * its n_local_min most recent ones, its U oldest tokens are clustered on their
 * own (as a segment of the build: same seeding rule with the segment's number,
 * same arithmetic) into min(k_u, U) clusters, which are appended to the index.
 * Nothing indexed before changes.  The result is written as a NEW index with
 * arrays of its own (this library's arrays are dense per unit, so an index with
 * more clusters has other strides); when no segment is flushed only the steady
 * rows differ from the old index.
 *
 * wave_index_append_plan (host only): fills *new_ix (dimensions, derived
 * fields; N = old N + n_new, n_local = what stays in the window), the byte
 * sizes of its nine buffers and the workspace wave_index_append needs.  An
 * index that already holds update segments takes the same U and k_u again.
 *
 * wave_index_append: old_ix read only; K_new, V_new DEVICE [B,Hkv,n_new,d]
 * dtype (may be NULL when n_new = 0); new_ix as planned, with its nine DEVICE
 * buffers (written; must not overlap old_ix's, with two exceptions: an update
 * which flushes no segment -- the plan's appended_segments equals the old one
 * -- may name old_ix's own seven arrays of the clustered part, which are then
 * left as they are; and perm, k_perm, v_perm may be old_ix's when both indexes
 * have the same row_capacity >= the new N_idx: the new rows are then written
 * behind the old ones in place and old_ix stays valid; centroids, vsum, sizes
 * and offsets may be old_ix's when both indexes have the same cluster_capacity
 * >= the new m: the new clusters are then written behind the old ones in place
 * (an update of 1K tokens then writes its 64 clusters and 1K rows per unit and
 * copies nothing that was indexed before; the new k_perm and v_perm rows are
 * working memory until the stream work completes, as in wave_index_build, the
 * old ones stay readable throughout); likewise k_steady and
 * v_steady may be old_ix's when no segment is flushed and both indexes have
 * the same steady_capacity >= the new p: only the new tokens' rows are then
 * written, behind the old window); workspace DEVICE, 256-byte aligned.  The
 * plan keeps old_ix's row_capacity, cluster_capacity and steady_capacity while
 * the grown index fits in them and reports 0 (dense) otherwise.  An array that
 * both indexes name must have the same stride per unit in both
 * (WAVE_ERR_ARG otherwise).  Errors: as wave_index_build; WAVE_ERR_SHAPE if new_ix is not the
 * plan of (old_ix, n_new, n_local_min, U, k_u) or old N < n_sink. */
wave_status wave_index_append_plan(const wave_index *old_ix, int n_new, int n_local_min,
                                   int update_segment_len, int update_clusters, wave_index *new_ix,
                                   size_t bytes[WAVE_INDEX_BUFFERS], size_t *workspace_bytes);
wave_status wave_index_append(const wave_index *old_ix, const void *K_new, const void *V_new,
                              int n_new, int n_local_min, int update_segment_len,
                              int update_clusters, int iters, uint64_t seed, wave_index *new_ix,
                              void *workspace, size_t workspace_bytes, void *hip_stream);

/* Index construction ("Index Organization", "Lightweight Index Construction"):
 * per unit and per segment of L tokens, spherical k-means on the centred,
 * unit-normalised keys (seeded distinct-point initialisation, `iters` rounds of
 * assign + update, ties to the lowest cluster id, empty clusters keep their
 * centroid; the partition is the one of the last assign); then per cluster its
 * size, the mean of its raw keys, the sum of its values, and the key/value rows
 * permuted so that clusters are contiguous.  Similarities are bf16 MFMA
 * products accumulated in fp32 (fp32 MFMA for f32 data); any point whose two
 * best similarities are closer than the accumulation error bound is re-decided
 * in fp64; centring, normalisation, centroid updates, means and value sums
 * accumulate in fp64 and are rounded once (to nearest even) to dtype.
 *   K, V       DEVICE [B,Hkv,N,d] dtype, read only, may be released after the
 *              stream work completes
 *   ix         dimensions + planned fields + the nine DEVICE buffers (written).
 *              The k_perm and v_perm rows are working memory of the k-means
 *              until the stream work completes: from the start of the call
 *              they hold nothing that another stream could read, and they must
 *              not overlap K or V
 *   workspace  DEVICE, 256-byte aligned, >= build_workspace_bytes
 * From the second round on, only clusters that a point entered or left get a
 * new centroid (the others keep theirs bit for bit); where the sums stay exact
 * in fp64 in any order, which is tested per segment, the points that moved are
 * taken out of one member sum and added to another, elsewhere the members are
 * summed again.  bf16 segments of
 * at most 2048 tokens and 128 clusters are clustered by one workgroup each that
 * runs all rounds; WAVE_NO_SMALL_KMEANS=1 in the environment keeps them on the
 * kernels of the long segments (same result, one launch per step). */
wave_status wave_index_build(const void *K, const void *V, wave_index *ix, int iters,
                             uint64_t seed, void *workspace, size_t workspace_bytes,
                             void *hip_stream);

/* One decode step of tripartite attention for B x Hq query heads (query head
 * hq uses the index of KV head hq / G and ranks clusters on its own):
 * score every non-empty centroid against q, take the topk_clusters best
 * (ties to the lower id), attend exactly over the steady tokens and over every
 * token of the selected clusters, let each other cluster contribute
 * s_i * exp(q.C_i / sqrt(d)) to the normaliser and exp(q.C_i / sqrt(d)) * VS_i
 * to the numerator (estimation equations), and merge the zones under one
 * softmax normalisation by log-sum-exp.
 *   q          DEVICE [B,Hq,d] dtype
 *   out        DEVICE [B,Hq,d] fp32; lse DEVICE [B,Hq] fp32 = log sum of
 *              exp(scaled logits) over the three zones (natural log)
 *   selected   DEVICE [B,Hq,topk_clusters] int32 or NULL: selected cluster ids
 *              ascending, padded with -1
 *   n_sink, n_local  must equal the index's, else WAVE_ERR_STEADY_MISMATCH
 *   topk_clusters >= number of non-empty clusters retrieves everything (the
 *   result is then exact attention); 0 leaves steady + estimation only.
 * Scores accumulate in fp32; a cluster whose fp32 score lies within the
 * accumulation error bound of the selection threshold is re-scored in fp64, so
 * the selected set is the fp64 ranking's (also when thousands of scores lie
 * inside that bound: they are then ranked in fp64 without being kept, slowly).
 * One exception: a head ranked by the streaming selection (more than 131072
 * clusters per KV head, or more than 2048 clusters passing the first-stage
 * filter of the many-cluster path) AND with more than 1024 scores inside the
 * bound keeps the fp32 ranking, ties to the lower id.
 *
 * Precondition on the index (it holds for every index this library builds or
 * grows; a caller that fills the arrays itself must keep it): each stored
 * centroid is the mean of the cluster's stored key rows and each stored value
 * sum the sum of its value rows, up to one rounding to dtype.  The estimation
 * terms are computed for ALL clusters in one pass over the meta index and the
 * selected clusters' terms are taken out again; by the estimation bound
 * (s_i exp(q.C_i / sqrt(d)) <= sum over the cluster's rows of exp(q.K_j /
 * sqrt(d)) when C_i is the mean) a term that is taken out never exceeds what
 * the cluster's exact rows put in, so the cancellation costs about one fp32
 * ulp of the result.  A centroid whose logit lies delta above that bound costs
 * about exp(delta) ulps (storage rounding of a bf16 centroid: delta <=
 * 2^-8 |q| |C_i| / sqrt(d), harmless); an index that breaks the bound grossly
 * loses the retrieved part of the result to cancellation.  If the normaliser
 * itself cancels to zero or below, out and lse of that head are NaN: never a
 * silent zero. */
wave_status wave_attention_decode(const void *q, const wave_index *ix, int Hq, int topk_clusters,
                                  int n_sink, int n_local, float *out, float *lse,
                                  int32_t *selected, void *workspace, size_t workspace_bytes,
                                  void *hip_stream);

/* wave_attention_decode for callers that cannot allocate device memory or hand a
 * workspace over: code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc.  Same arguments, results and kernels as
 * wave_attention_decode, without the workspace: the step's scratch (scores,
 * selected ids, partial results) lives in a static device array of
 * WAVE_STATIC_SCRATCH_BYTES inside the library, which every GPU the library
 * runs on holds from the first call on it until the process ends.  The call
 * allocates and frees nothing.  A step whose scratch would not fit (the size is
 * what wave_index_plan reports as decode_workspace_bytes) is refused with
 * WAVE_ERR_WORKSPACE before anything is launched; the five benchmark workloads
 * fit (the largest, 64 sequences x 28 query heads x 4096 clusters, needs 47 MB).
 * All calls on one GPU share the one array: calls that overlap in time on the
 * same GPU (two streams, two threads) race; order them on one stream or by
 * events.  Nothing in the array has to be zero when a step starts, so nothing is
 * cleared between calls.  wave_attention_decode_static_capacity returns
 * WAVE_STATIC_SCRATCH_BYTES. */
#define WAVE_STATIC_SCRATCH_BYTES (64u << 20)
size_t wave_attention_decode_static_capacity(void);
wave_status wave_attention_decode_static(const void *q, const wave_index *ix, int Hq,
                                         int topk_clusters, int n_sink, int n_local, float *out,
                                         float *lse, int32_t *selected, void *hip_stream);

/* The decode step with a budget for the estimation zone, as in the paper's
 * evaluation (parameter paragraph: an estimation zone of 23.2 % of the clusters
 * so that the three zones cover about a quarter of the context) and its
 * ablation without estimation: of the clusters that are not retrieved, only the
 * est_clusters best-scoring ones (same ranking and tie rule as the retrieval)
 * enter through their centroid, size and value sum; the others are ignored.
 * est_clusters < 0, or a budget that reaches every cluster, is
 * wave_attention_decode itself; est_clusters = 0 leaves the exact zones only.
 * Same arguments otherwise; the workspace size comes from
 * wave_attention_decode_budget_workspace (0 if the arguments are invalid).
 * Up to 65536 clusters per KV head it runs in four launches (scores with the
 * steady zone, both selections at once, retrieval with estimation, merge);
 * beyond that its steps are launches of their own.  Every head reads its own
 * estimated clusters' value sums, so a budget moves about as many bytes as
 * estimating every cluster once per KV head and is not faster than
 * wave_attention_decode. */
size_t wave_attention_decode_budget_workspace(const wave_index *ix, int Hq, int topk_clusters,
                                              int est_clusters);
wave_status wave_attention_decode_budget(const void *q, const wave_index *ix, int Hq,
                                         int topk_clusters, int est_clusters, int n_sink,
                                         int n_local, float *out, float *lse, int32_t *selected,
                                         void *workspace, size_t workspace_bytes, void *hip_stream);

/* Full decode attention, the operation the wave index approximates (the
 * attention equation of the background section): for every query head,
 * o = softmax(q K^T / sqrt(d)) V over all N tokens of its KV head, by streaming
 * K and V once per KV head with an online softmax (fp32 accumulation) and one
 * log-sum-exp merge.  It is the same-hardware baseline for the decode step and
 * the limit wave_attention_decode reaches when every cluster is retrieved.
 *   q          DEVICE [B,Hq,d] dtype;  K, V  DEVICE [B,Hkv,N,d] dtype
 *   out        DEVICE [B,Hq,d] fp32;   lse   DEVICE [B,Hq] fp32 (natural log)
 *   workspace  DEVICE, 256-byte aligned, >= wave_full_attention_workspace(...)
 * wave_full_attention_workspace returns 0 for unsupported shapes. */
size_t wave_full_attention_workspace(int B, int Hq, int N, int d);
wave_status wave_full_attention_decode(const void *q, const void *K, const void *V, int dtype, int B,
                                       int Hq, int Hkv, int N, int d, float *out, float *lse,
                                       void *workspace, size_t workspace_bytes, void *hip_stream);

/* ---------------------------------------------------------------------------
 * The plain cache: rotary positions, and one cache of raw rows per sequence
 * that grows token by token, is attended exactly (alone or behind a prefix that
 * the whole batch shares) and is kept at a budget by what its rows are worth.
 * It holds what no index holds: the tokens of ragged conversations, read by
 * the same decode conventions (q, out, lse) as above, so that its lse merges
 * with that of any other zone.
 * ------------------------------------------------------------------------- */

/* Rotary positions with 1 .. WAVE_ROTARY_MAX_AXES axes.  The first rot_dim
 * channels of a row form rot_dim / 2 pairs, the others stay as they are.  Pair
 * i of a token turns by the angle coordinate[axis[i]] * inv_freq[i]:
 *   (x, y) -> (x cos - y sin, x sin + y cos).
 * Plain data: wave_rotary_plan fills it, and a caller with frequencies of its
 * own (a scaled or a learned ladder) writes them into inv_freq afterwards. */
enum { WAVE_ROTARY_MAX_AXES = 4, WAVE_ROTARY_MAX_PAIRS = 64 };
typedef enum {
  WAVE_ROTARY_RUNS = 0,    /* axis 0 has the first sections[0] pairs, axis 1 the next, ... */
  WAVE_ROTARY_TURNS = 1,   /* pairs dealt out in turn: axis 0, 1, .., 0, 1, .. while an axis has some left */
  WAVE_ROTARY_LADDERS = 2  /* as runs, and the frequencies of every axis start anew */
} wave_rotary_order;
typedef enum {
  WAVE_ROTARY_HALVES = 0,   /* pair i: channels i and i + rot_dim / 2 */
  WAVE_ROTARY_NEIGHBOURS = 1 /* pair i: channels 2 i and 2 i + 1      */
} wave_rotary_pairing;
typedef struct {
  int32_t rot_dim;          /* rotated channels: a multiple of 16, at most d           */
  int32_t n_axes;
  int32_t pairing;          /* wave_rotary_pairing                                     */
  int32_t axis[WAVE_ROTARY_MAX_PAIRS];     /* axis of each pair, < n_axes              */
  double inv_freq[WAVE_ROTARY_MAX_PAIRS];  /* radians per position of each pair        */
} wave_rotary;

/* Host only.  sections: HOST [n_axes], pairs of each axis, adding up to
 * rot_dim / 2 (an axis may have none).  inv_freq[i] = base^(-i / (rot_dim / 2)),
 * with WAVE_ROTARY_LADDERS base^(-i' / sections[a]) for the i'-th pair of axis a.
 * WAVE_ERR_SHAPE: rot_dim not a multiple of 16 in 16 .. 128, or sections that do
 * not add up; WAVE_ERR_ARG: anything else (base must be finite and > 0). */
wave_status wave_rotary_plan(wave_rotary *rotary, int rot_dim, double base, const int32_t *sections,
                             int n_axes, int order, int pairing);

/* Rotates x into y.
 *   x, y       DEVICE [B,H,N,d] dtype, 16-byte aligned; y may be x, and must not
 *              overlap it otherwise
 *   coords     DEVICE [n_axes,B,N] int32, any values; must not overlap y
 * Angles are formed in fp64 (their error is about 2^-53 of the angle, so positions of a million
 * are as exact as small ones), sine and cosine and the products in fp32, and
 * each result is rounded once to dtype.  H and N may be anything from 1 to 2^30
 * (B * H and B * N below 2^31).  A turn's gradient is the turn back: the same call with the
 * inv_freq negated. */
wave_status wave_rotary_apply(const void *x, const int32_t *coords, const wave_rotary *rotary, int dtype,
                              int B, int H, int N, int d, void *y, void *hip_stream);

/* Rows of several heads where they lie: element c of the row of sequence b, head h and token n is
 * data[b * stride_b + h * stride_h + n * stride_n + c], so a fused projection's output is read without a
 * copy.  Strides are in elements, none negative (0 repeats a row), each a multiple of 16 bytes;
 * data is 16-byte aligned. */
typedef struct {
  const void *data;         /* DEVICE dtype                                            */
  int64_t stride_b, stride_h, stride_n;
} wave_rows;

/* Norms of queries and keys for each head: row x becomes x_c * weight_c / sqrt(mean(x^2) + eps), the mean over all d
 * channels, before it is turned. */
typedef struct {
  const void *q_weight, *k_weight; /* DEVICE [d] dtype, 16-byte aligned; NULL: those rows are not normed */
  float eps;                       /* 0 or more, finite                                */
} wave_head_norm;

/* Norms and rotary positions of queries and keys in one pass.
 *   q, k       rows [B,Hq,N] and [B,Hkv,N]; either may be NULL (its heads and output are then not looked at)
 *   norm       HOST, or NULL: nothing is normed
 *   rotary     HOST, or NULL: nothing is turned; coords must then be NULL, and norm must not
 *   coords     DEVICE [n_axes,B,N] int32
 *   q_out, k_out  DEVICE [B,Hq,N,d] and [B,Hkv,N,d] dtype, dense, 16-byte aligned; each may be its own input
 *              where that is dense, and must not overlap anything else that the call reads or writes
 * Sums of squares, norms, sines and products are fp32 and each result is rounded once to dtype: a row whose squares add
 * up to 2^128 and more has norm infinity, squares below 2^-149 count as 0.  Angles are those of wave_rotary_apply, their sines and
 * cosines nearer than there (to a last place, there to 2^-22), so a turned row may have other last bits than that call's.
 * Sizes as in wave_rotary_apply, with H = Hq + Hkv. */
wave_status wave_norm_rotary_apply(const wave_rows *q, int Hq, const wave_rows *k, int Hkv,
                                   const wave_head_norm *norm, const wave_rotary *rotary,
                                   const int32_t *coords, int dtype, int B, int N, int d, void *q_out,
                                   void *k_out, void *hip_stream);

/* One cache of raw key and value rows per (sequence, KV head).  Plain data, all
 * arrays caller-owned; a field that a call does not need may be NULL.  Rows of
 * sequence b are the first lengths[b] of each of its units, in no order that
 * matters; what lies behind them is never read and may hold anything.  The
 * library reads lengths on the device: a value outside 0 .. capacity counts as
 * the nearer of the two.  Every call returns WAVE_ERR_SHAPE for B * Hkv of 2^21
 * and more or a capacity above 2^30. */
typedef struct {
  int32_t dtype;            /* wave_dtype                                              */
  int32_t B, Hkv, d;
  int32_t capacity;         /* rows allocated per unit                                 */
  void *k, *v;              /* DEVICE [B,Hkv,capacity,d] dtype, 16-byte aligned        */
  int32_t *positions;       /* DEVICE [B,Hkv,capacity] number of each row's token in   */
                            /*        its sequence                                     */
  float *weights;           /* DEVICE [B,Hkv,capacity] attention weight received so far */
  int32_t *lengths;         /* DEVICE [B] rows in use                                  */
  int32_t *tokens;          /* DEVICE [B] tokens appended so far, evicted ones too     */
} wave_cache;

/* Appends n_new tokens (1 for a decode step, any number for a prompt) to every sequence:
 * keys and queries are rotated as by wave_rotary_apply, and token t of sequence
 * b becomes row lengths[b] + t of its units, with position tokens[b] + t and
 * weight 0.  q is only rotated; it may be used by wave_cache_attention_decode
 * as it is where n_new = 1.
 *   k_new, v_new  DEVICE [B,Hkv,n_new,d] dtype
 *   q             DEVICE [B,Hq,n_new,d] dtype or NULL (then Hq and q_out are not
 *                 looked at); q_out the same shape, may be q
 *   counts        DEVICE [B] int32 or NULL: only the first counts[b] of the n_new
 *                 tokens exist (a padded batch; a value outside 0 .. n_new counts as
 *                 the nearer); nothing of the others is written, their rows of
 *                 q_out included
 *   rotary        HOST, or NULL: keys go in as they are; q must then be NULL
 *   coords        DEVICE [n_axes,B,n_new] int32, or NULL: tokens[b] + t on every axis.
 *                 Must not overlap what the call writes (the cache's k, v, positions and
 *                 weights, q_out, lengths_out, tokens_out), except that with one axis and
 *                 n_new = 1 it may be cache->lengths or cache->tokens themselves, updated
 *                 in place
 *   lengths_out, tokens_out  DEVICE [B]: the numbers after the call.  Each may be
 *                 the cache's own array (updated in place) and must not overlap it
 *                 otherwise; tokens_out may be NULL where cache->tokens is.
 * cache->positions, weights and tokens may be NULL (positions and NULL coords
 * need tokens).  What the call writes must not overlap what it reads or writes otherwise.
 * The caller keeps lengths[b] + counts[b] <= capacity: rows that
 * do not fit are left out, and lengths and tokens advance by those that did.
 * WAVE_ERR_SHAPE: n_new above 2^30, B * n_new of 2^31 and more, B * Hq of 2^24
 * and more. */
wave_status wave_cache_append(const wave_cache *cache, const void *k_new, const void *v_new, const void *q,
                              int Hq, int n_new, const int32_t *counts, const wave_rotary *rotary,
                              const int32_t *coords, void *q_out, int32_t *lengths_out,
                              int32_t *tokens_out, void *hip_stream);

/* Exact attention of one token per sequence over a prefix that all sequences
 * share and the sequence's own rows, under one softmax:
 *   o = softmax([q Kp^T, q K_b^T] / sqrt(d)) [Vp; V_b].
 * The prefix is read once for the batch (all B * G queries of a KV head
 * multiply the same rows), the own rows once per KV head.
 *   q             DEVICE [B,Hq,d] dtype, 16-byte aligned
 *   prefix_k, prefix_v  DEVICE [Hkv,P,d] dtype, dense (the k and v of a cache with B = 1
 *                 and capacity = P are), 16-byte aligned; may be NULL where P = 0
 *   weights_out   DEVICE [B,Hkv,capacity] fp32 or NULL.  Each own row j of a unit
 *                 gets decay * weights[j] + the sum over the unit's G heads of the
 *                 softmax weight that row j received (the prefix's share counts in
 *                 the normaliser).  May be cache->weights, and must not overlap it
 *                 otherwise; rows behind the length are left as they are.  decay in
 *                 0 .. 1; with 0 the old weights are not read
 *   out           DEVICE [B,Hq,d] fp32;  lse DEVICE [B,Hq] fp32 (natural log); they and
 *                 weights_out need no more than the alignment of a float
 *   workspace     DEVICE, 256-byte aligned, >= wave_cache_attention_workspace(...);
 *                 what a longer prefix, a larger capacity or accumulate = 1 needs is
 *                 enough for a shorter one, a smaller one and accumulate = 0
 * A sequence with neither prefix nor own rows has out = 0 and lse = -infinity.
 * Scores are exact products of the stored values, summed in fp32; the softmax and
 * all sums are fp32.  For bf16 caches a softmax weight meets the values as three
 * bf16 numbers that hold all its bits.
 * A value that is infinite or no number makes its channel of every head that
 * attends to its row one or the other.
 * WAVE_ERR_SHAPE: Hq / Hkv not a whole number in 1 .. 8, P above 2^30, or
 * B * Hq + B * Hkv * ceil(capacity / 1024) of 2^24 and more. */
size_t wave_cache_attention_workspace(const wave_cache *cache, int Hq, int P, int accumulate);
wave_status wave_cache_attention_decode(const void *q, int Hq, const wave_cache *cache,
                                        const void *prefix_k, const void *prefix_v, int P, float decay,
                                        float *weights_out, float *out, float *lse, void *workspace,
                                        size_t workspace_bytes, void *hip_stream);

/* Eviction by accumulated attention weight: every unit of a sequence with more
 * than n_keep rows keeps n_keep of them.  Rows whose position is below n_sink or
 * among the last n_local of the sequence's tokens come first, then the rows of
 * the largest weight; equal ones: the lower row first; a weight that is not a number
 * counts as less than any other.  A kept row below n_keep stays where it is; the
 * i-th kept row from n_keep on moves to the i-th row below it that left.  So in
 * place only the moved rows are read and written, and the order of the rows
 * changes: positions says which is which.
 *   from          the cache (weights, positions, tokens and lengths are needed)
 *   to            what it becomes: to->k and to->v are from's own (in place) or
 *                 other arrays (all kept rows are written there, e.g. into a
 *                 smaller cache); the same choice, each on its own, for positions,
 *                 weights, lengths and tokens.  An array that both name needs the same
 *                 capacity, others must not overlap.  to->capacity >= min(n_keep,
 *                 from->capacity).  Rows behind the new length are left as they are
 *   n_sink + n_local <= n_keep (WAVE_ERR_ARG otherwise)
 *   (WAVE_ERR_SHAPE also where 64 GiB of keys and more may be written: B * Hkv * (rows * bytes of a row / 4096 + 1)
 *   of 2^24 and more, rows = min(n_keep, capacity - n_keep) in place and n_keep into other arrays)
 *   workspace     DEVICE, 256-byte aligned, >= wave_cache_evict_workspace(...) */
size_t wave_cache_evict_workspace(const wave_cache *from, int n_keep);
wave_status wave_cache_evict(const wave_cache *from, const wave_cache *to, int n_keep, int n_sink,
                             int n_local, void *workspace, size_t workspace_bytes, void *hip_stream);

/* ---------------------------------------------------------------------------
 * The paged cache: keys and values in 8 bits, in pages that sequences share.
 * A page holds `page` tokens of every KV head.  New rows wait in the sequence's
 * tail, in dtype; as soon as a page's last row is there the page is rounded to 8
 * bits, once, with one scale for each head, and never changes again: what a page holds does
 * not depend on how its tokens came in, the newest rows are exact, and sequences that begin
 * alike share pages.
 *   scale = max |x| / 127 over the page's rows of a head, as they are in dtype;
 *   code  = x * ((1 / max |x|) * 127) to the nearest whole number, ties to even (fp32, each step rounded)
 * and a row reads as code * scale.  A head's part of a page whose largest value is below 2^-100 reads as zeros
 * (scale 0); one that holds an infinity or no number reads as no numbers throughout.
 *
 * Plain data, all arrays caller-owned.  A sequence of L tokens has L / page pages, the first entries of its row of
 * the table, and L % page rows in its tail; what lies behind either is never read.
 * references counts the sequences that hold a page; one with 0 (or less) is free, so an empty
 * cache is lengths and references of 0.  A caller who keeps a page (a prompt that comes back) adds 1 of its own.
 * A sequence is not cut short by setting its length back: the rows of a complete page are no longer in the tail.
 * Appends to, and reorderings of, states of one pool take and give back the same pages: the caller orders them, and goes
 * on with the state that the last one left.  What only reads a state may run beside an append that leaves it as it is.
 * The library reads lengths and table on the device: a length outside 0 ..
 * max_pages * page + page - 1 and an entry outside 0 .. n_pages - 1 count as the nearest inside.
 * max_pages and n_pages also choose between forms of a call, as lengths are the device's: short sequences have their fastest
 * attention, reordering and appended token in a table and a pool that are not much larger than they need.
 * Every call returns WAVE_ERR_SHAPE for a page other than 32, 64 or 128, B * Hkv of 2^21 and more,
 * n_pages above 2^28, or max_pages * page above 2^30.
 * ------------------------------------------------------------------------- */
typedef struct {
  int32_t dtype;            /* wave_dtype of queries, new rows and tails               */
  int32_t B, Hkv, d;
  int32_t page;             /* tokens of a page: 32, 64 or 128                         */
  int32_t n_pages;          /* pages of the pool                                       */
  int32_t max_pages;        /* entries of a sequence's row of the table                */
  int8_t *k_codes, *v_codes;  /* DEVICE [n_pages,Hkv,page,d], 16-byte aligned          */
  float *k_scales, *v_scales; /* DEVICE [n_pages,Hkv]                                  */
  void *k_tail, *v_tail;    /* DEVICE [B,Hkv,page,d] dtype, 16-byte aligned            */
  int32_t *table;           /* DEVICE [B,max_pages] pages of each sequence             */
  int32_t *lengths;         /* DEVICE [B] tokens                                       */
  int32_t *references;      /* DEVICE [n_pages]                                        */
} wave_pages;

/* Appends n_new tokens (1 for a decode step, any number for a prompt) to every sequence: keys and queries are
 * normed and turned as by wave_norm_rotary_apply, rows are rounded to dtype, and every page that becomes complete takes a
 * free page of the pool: the lowest ones, in the order of the sequences and of each sequence's tokens.
 *   from          the cache (every array is needed)
 *   to            what it becomes: k_tail, v_tail, table, lengths and references are all from's own (in
 *                 place) or all other arrays, and from is then still what it was, so an append of drafted tokens
 *                 is taken back by going on with from.  (Then only one of the two may go on: both count the same
 *                 pages as free.)  Codes and scales are from's own, and so are all sizes.  What lies behind a
 *                 sequence's pages and rows in to's arrays is left as it is
 *   k_new, v_new  rows [B,Hkv,n_new]
 *   q             rows [B,Hq,n_new] or NULL (then Hq and q_out are not looked at); only normed and turned.
 *                 q_out DEVICE [B,Hq,n_new,d] dtype, may be q where that is dense.  NULL where there is neither a
 *                 rotary plan nor norm->q_weight
 *   counts        DEVICE [B] int32 or NULL: only the first counts[b] of the n_new tokens exist (a value
 *                 outside 0 .. n_new counts as the nearer); nothing of the others is written, their rows
 *                 of q_out included
 *   norm, rotary  HOST, or NULL
 *   coords        DEVICE [n_axes,B,n_new] int32, or NULL: lengths[b] + t on every axis
 *   workspace     DEVICE, 256-byte aligned, >= wave_pages_append_workspace(from)
 * Tokens that do not fit, in the table's row or because no page is free for them, are left out (their rows of q_out are
 * written): a sequence then ends one row before the page that it did not get, and lengths
 * says how many there are.  What the call writes must not overlap what it reads or writes otherwise.
 * WAVE_ERR_SHAPE: n_new above 2^30, B * n_new of 2^31 and more, B * Hq of 2^24 and more; queries that are turned without
 * coords where a token's number could pass 2^31 - 1: max_pages * page + page - 1 + n_new above 2^31. */
size_t wave_pages_append_workspace(const wave_pages *from);
wave_status wave_pages_append(const wave_pages *from, const wave_pages *to, const wave_rows *k_new,
                              const wave_rows *v_new, const wave_rows *q, int Hq, int n_new,
                              const int32_t *counts, const wave_head_norm *norm, const wave_rotary *rotary,
                              const int32_t *coords, void *q_out, void *workspace, size_t workspace_bytes,
                              void *hip_stream);

/* Rows back in dtype (an index is built from raw rows): row t of the outputs is row first[b] + t of sequence b, pages'
 * rows rounded once; rows that the sequence has not are left as they are.
 *   first         DEVICE [B] int32, or NULL: 0
 *   k_out, v_out  DEVICE [B,Hkv,n,d] dtype, 16-byte aligned; one may be NULL
 * (references is not needed.)  WAVE_ERR_SHAPE: n above 2^30, or B * Hkv * n of 2^34 and more. */
wave_status wave_pages_read(const wave_pages *pages, const int32_t *first, int n, void *k_out, void *v_out,
                            void *hip_stream);

/* Exact attention of one token per sequence over the rows that the cache holds: o = softmax(q K_b^T / sqrt(d)) V_b.
 *   q             DEVICE [B,Hq,d] dtype, 16-byte aligned
 *   out           DEVICE [B,Hq,d] fp32;  lse DEVICE [B,Hq] fp32 (natural log)
 *   workspace     DEVICE, 256-byte aligned, >= wave_pages_attention_workspace(...)
 * A sequence without rows has out = 0 and lse = -infinity.  Scores are exact products of queries and codes, summed in fp32,
 * times the page's scale; the softmax and all sums are fp32, and a softmax weight meets the values' codes as three bf16
 * numbers that hold all its bits.  Sums are divided by the normaliser at their end, over weights of up to 2^8: they are no numbers where 2^8
 * times a sequence's rows times its largest value passes 2^128, or d * 127 times the largest channel of a query does.
 * (references is not needed.)
 * WAVE_ERR_SHAPE: Hq / Hkv not a whole number in 1 .. 8, or B * Hq of 2^24 and more. */
size_t wave_pages_attention_workspace(const wave_pages *pages, int Hq);
wave_status wave_pages_attention_decode(const void *q, int Hq, const wave_pages *pages, float *out, float *lse,
                                        void *workspace, size_t workspace_bytes, void *hip_stream);

/* Sequences copied, forked and freed: sequence b of `to` becomes what sequence parent[b] of `from` was, an empty one where
 * parent[b] is outside 0 .. from->B - 1.  Pages are shared, so only tables and tails are copied; references changes by
 * what `to` holds of each page less what `from` held.
 *   parent        DEVICE [to->B] int32
 *   to            k_tail, v_tail, table, lengths and references are all other arrays (B may then be
 *                 another; from is still what it was, but only one of the two may go on), or all from's
 *                 own: then a sequence can only stay, parent[b] = b, or leave, any other number.
 *                 Codes and scales are from's own (the call does not touch them) */
wave_status wave_pages_reorder(const wave_pages *from, const wave_pages *to, const int32_t *parent,
                               void *hip_stream);

/* Test hook, host only: the k_s distinct seed-token indices (relative to the
 * segment start) with which segment s of unit (b, h) starts k-means: the first
 * k_s entries of a Fisher-Yates shuffle of 0..L_s-1 driven by splitmix64 keyed
 * on (seed, b, h, s).  out: HOST [k_s]. */
wave_status wave_init_indices(uint64_t seed, int b, int h, int s, int L_s, int k_s, int32_t *out);

/* Test hook: one assign step of the build on one segment, with the build's
 * own kernels.  xhat DEVICE [L_s,d] dtype (normalised keys), chat DEVICE
 * [k_s,d] dtype (centroids), assign DEVICE [L_s] int32 (written).
 * workspace DEVICE >= 4*L_s + 1024 bytes, 256-byte aligned. */
wave_status wave_kmeans_assign_step(const void *xhat, const void *chat, int dtype, int L_s, int k_s,
                                    int d, int32_t *assign, void *workspace,
                                    size_t workspace_bytes, void *hip_stream);

/* Calibration: plain streaming kernels over a buffer of known size, for the
 * callers that measure (the benchmark and profiler runs): a profiler counter read
 * for them gives the factor between its unit and bytes, and their rate is the
 * bandwidth a simple kernel reaches on the machine.  src, dst DEVICE, 16-byte
 * aligned, `bytes` a multiple of 16; `workgroups` of 256 threads stride over the
 * buffer.  copy reads src and writes dst; read only reads src (sink: DEVICE, at
 * least 4 bytes, practically never written). */
wave_status wave_calibration_copy(void *dst, const void *src, size_t bytes, int workgroups,
                                  void *hip_stream);
wave_status wave_calibration_read(const void *src, size_t bytes, void *sink, int workgroups,
                                  void *hip_stream);

/* Profiler (the library's only global state).  While enabled, every kernel the
 * library launches is bracketed by HIP events on its stream.
 * wave_profile_read synchronises, adds up the elapsed time per kernel name
 * since the last read and writes up to `cap` entries: names[i] points to a
 * static string, total_ms[i] and launches[i] to the sums.  Returns the number
 * of distinct kernels, or -1 on a HIP error. */
wave_status wave_profile_enable(int on);
int wave_profile_read(const char **names, float *total_ms, int *launches, int cap);

const char *wave_status_string(wave_status st);

#ifdef __cplusplus
}
#endif
#endif /* WAVE_H */
