/*
 * libpasa -- PASA (online pseudo-average shifting attention, arXiv 2503.01873) forward pass for
 * AMD MI355X (gfx950).  C ABI: plain pointers and sizes, no C++ types, no exceptions.
 *
 * What is computed (paper section 1.1 problem statement, Algorithm 1):
 *     O = softmax(scale * Q K^T) V      per (batch, query head), optionally causal,
 * evaluated FlashAttention-style over key tiles of 128 keys.  Each key tile is shifted by beta times
 * its own mean along the sequence and scaled (Eq. (10), (11)), which leaves every softmax row unchanged
 * (Eq. (9)); a per-row global recovering step re-aligns the running maximum, sum and output across
 * tiles (Eq. (13)-(15), Algorithm 1 steps 1-4) so that half-precision scores stay far below 65504.
 * N need not be a multiple of 128: a ragged last tile uses its own key count as the divisor of the tile
 * mean and of the pseudo-average, which keeps Eq. (14) valid for it (the paper does not state this case).
 *
 * Layouts.  q, o: [B, Hq, N, d];  k, v: [B, Hkv, N, d].  IEEE fp16 (or bf16, see pasa_io_dtype), row-major, contiguous, DEVICE
 * pointers, 16-byte aligned.  Query head h reads KV head h / (Hq / Hkv) (grouped-query attention; the
 * paper does not discuss it).  causal != 0: key n is visible to query r iff n <= r.
 *
 * Ownership.  The caller owns every buffer, including the workspace.  The library keeps no device
 * state between calls.  q, k, v are only read; o is only written and must not alias an input.
 *
 * Streams.  `stream` is a hipStream_t passed as void* (NULL = the default stream).  Every entry point
 * only enqueues work and returns; it never synchronises the device.
 *
 * Errors.  Every function returning int returns a pasa_status.  All argument checking happens on the
 * host before anything is enqueued; on error nothing has been launched.
 */
#ifndef PASA_H
#define PASA_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PASA_OK = 0,
    PASA_EINVAL = 1,       /* null or misaligned pointer, non-positive size, Hq % Hkv != 0, bad scale / beta / variant */
    PASA_EUNSUPPORTED = 2, /* d not in {64, 128}, a length > 262144, shift_tile != 128, PASA_SHIFT_MATRIX with N % 128 != 0 */
    PASA_ELAUNCH = 3,      /* the HIP runtime refused an allocation or a launch */
    PASA_EWORKSPACE = 4    /* workspace missing, misaligned or smaller than pasa_attn_fwd_workspace() */
} pasa_status;

/* Precision allocation of the tile loop (paper section 1.2).  The matrix cores always accumulate in
 * fp32; "fp16" below means the value is rounded to fp16 (nearest-even) where Algorithm 1 marks it. */
typedef enum {
    PASA_MIXED = 0,    /* K' and P fp16 (the GEMM operands); S', row statistics and O fp32 */
    PASA_STRICT16 = 1, /* Algorithm 1 as printed: S', P, Sbar', F, all Delta terms, m, l, P V and O rounded to fp16 */
    PASA_NAIVE16 = 2,  /* no shift (beta forced to 0): raw S = Q K^T rounded to fp16, then scaled; rest fp32.
                          This is the partially low-precision FlashAttention that overflows (section 2.1, Table 4). */
    PASA_S16 = 3,      /* shifted like MIXED, S' rounded to fp16 as it leaves the matrix core, statistics and O fp32 */
    PASA_DIRECT = 4    /* NOT the paper's recovering step ("direct-bias recovery").  Same idea of a shifted K' so that the
                          scores stay small, precision allocation of MIXED, but the shift vector of a tile is the fp16
                          vector k0 = fp16(beta * mean_tile(K)), K' = fp16((K - k0) * scale), and the removed bias is
                          added back as scale * (q . k0) (legal by Eq. (9): any shift leaves softmax unchanged)
                          followed by ordinary online softmax (Eq. (4)-(8)).  There is no pseudo-average Sbar' and no
                          factor beta/(1-beta), so the rounding noise of K' is not amplified.  The other shift modes do
                          not apply to it. */
} pasa_variant;

/* How the key pre-processing loop of Algorithm 1 forms K' (Eq. (10), (11)). */
typedef enum {
    PASA_SHIFT_MEAN = 0,   /* K' = fp16((K - beta * mean_tile(K)) * scale): mean by reduction in fp64, one rounding.
                              The shifting matrix is never formed, so its entries are never rounded. */
    PASA_SHIFT_MATRIX = 1, /* Algorithm 1 as printed: K'^T = K^T M with every entry of M = I/alpha - beta J/(128 alpha),
                              alpha = 1/scale, rounded to fp16 first (the rounding that section 2.3 and Eq. (20)-(22)
                              analyse); the product is exact (fp64) and rounded to fp16 once.  Evaluated as
                              (a - b) K + b sum_tile(K) with a, b the rounded diagonal and off-diagonal entry, which
                              is the same contraction.  Needs N % 128 == 0. */
    PASA_SHIFT_MATRIX_MFMA = 2 /* The same product as a batched GEMM on the matrix core, the way Algorithm 1's pre-processing
                              loop prints it: v_mfma_f32_32x32x16_f16 with K^T and the rounded M as operands, the 128
                              products of an output accumulated in fp32, one rounding to fp16.  Differs from
                              PASA_SHIFT_MATRIX by the fp32 accumulation only (a fraction of a per cent of the K' values
                              land on the neighbouring fp16 value).  Needs N % 128 == 0; not combined with the adaptive
                              entry point. */
} pasa_shift_mode;

/* Element type of q, k, v and o.  The method computes in fp16: bf16 inputs are converted to fp16 as they are loaded
 * (round to nearest even; magnitudes beyond 65504 become infinities), as the paper prescribes for BF16 inputs, and
 * the output is rounded to bf16 when it is stored. */
typedef enum { PASA_IO_F16 = 0, PASA_IO_BF16 = 1 } pasa_io_dtype;

typedef struct {
    float beta;        /* shift fraction of Eq. (10).  < 0: library default -- by mean 63.5/64.5 (invariance beta/(1-beta) =
                          63.5, the fp16 value of the invariance of the paper's adopted beta), by matrix the paper's
                          adopted beta = 0.984497 (Table 3);  0: plain FlashAttention;  otherwise must lie in [0, 1). */
    int variant;       /* a pasa_variant */
    int shift_tile;    /* keys per pseudo-average group; 0 or 128 (the only supported size) */
    unsigned long long* overflow_s;  /* optional DEVICE counter (caller zeroes it): score-tile entries whose magnitude
                                        exceeds 65504 where they would be stored as fp16.  NULL: not counted.
                                        A call with either counter runs on the 256-row kernel, which counts: its output
                                        agrees with that of the call without them up to rounding. */
    unsigned long long* nonfinite_o; /* optional DEVICE counter (caller zeroes it): inf/NaN entries written to o. */
    int shift_mode;    /* a pasa_shift_mode */
    int io_dtype;      /* a pasa_io_dtype; applies to q, k, v, o of the call it is passed to (the workspace is always
                          fp16, so pasa_prepare_kv and the calls that use its workspace may differ in it) */
} pasa_opts;

/* Default configuration: PASA_MIXED, default beta.  Allocates and frees its workspace in stream order
 * (hipMallocAsync / hipFreeAsync).  scale multiplies Q K^T (normally 1/sqrt(d)); finite and > 0. */
int pasa_attn_fwd(const void* q, const void* k, const void* v, void* o,
                  int B, int Hq, int Hkv, int N, int d, int causal, float scale, void* stream);

/* Bytes of device workspace pasa_attn_fwd_ex needs for these sizes: shifted keys K' and re-tiled values, both fp16
 * (4*B*Hkv*ceil(N/128)*128*d bytes), then one fp16 shift vector per key tile (2*B*Hkv*ceil(N/128)*d bytes, rounded up
 * to a multiple of 256; written by PASA_DIRECT's pre-processing, in plain order), then one 64-bit counter per (batch, KV head) (8*B*Hkv
 * bytes, rounded up to a multiple of 256; used by pasa_attn_fwd_adaptive only), then for every (batch, KV head) and
 * group of 16 key tiles the per-channel means of the rounded K' of those tiles as fp16 pairs (64*d bytes per group,
 * B*Hkv*ceil(ceil(N/128)/16) groups; PASA_MIXED takes the pseudo-average of Eq. (14) as the query times that mean,
 * Eq. (12); for PASA_DIRECT the same blocks hold the tiles' shift vectors k0 instead); these regions together are pasa_attn_fwd_workspace_min().  Last comes the
 * region of the key split: when a call would leave compute units idle, the keys of every workgroup are divided among
 * several workgroups, each of which leaves per query row its unnormalised output (d floats) and two doubles (running sum, level), and a second
 * kernel merges them with the log-sum-exp rule (the same algebra that lets the method run as ring attention, section
 * 2.2).  The region is sized for a call with N query rows (at least 1 MiB, so that short query chunks can split);
 * a call given less than that splits fewer ways or not at all, and one given less than pasa_attn_fwd_workspace_min()
 * fails with PASA_EWORKSPACE.  Not used by PASA_STRICT16 (its fp16 state has no merge rule in Algorithm 1) nor by the
 * adaptive entry point.  Returns 0 if the sizes are invalid. */
size_t pasa_attn_fwd_workspace(int B, int Hq, int Hkv, int N, int d);

/* The part of the workspace every call needs (all regions but the key split's). */
size_t pasa_attn_fwd_workspace_min(int B, int Hkv, int N, int d);

/* As pasa_attn_fwd, with options and a caller-provided workspace (DEVICE pointer, 256-byte aligned,
 * pasa_attn_fwd_workspace() bytes -- at least pasa_attn_fwd_workspace_min(); contents on return are unspecified).  opts == NULL means
 * {beta = -1, PASA_MIXED, 128, NULL, NULL, PASA_SHIFT_MEAN, PASA_IO_F16}.  Performs no allocation. */
int pasa_attn_fwd_ex(const void* q, const void* k, const void* v, void* o,
                     int B, int Hq, int Hkv, int N, int d, int causal, float scale,
                     const pasa_opts* opts, void* workspace, size_t workspace_bytes, void* stream);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc): pasa_attn_fwd_ex with its workspace in a fixed array of PASA_STATIC_WORKSPACE_BYTES of
 * device memory that belongs to the library (one copy per GPU the library is used on, held until the process ends).
 * Calls no hipMalloc / hipFree and no allocating routine.  PASA_EWORKSPACE if
 * pasa_attn_fwd_workspace_min(B, Hkv, N, d) exceeds PASA_STATIC_WORKSPACE_BYTES (e.g. B*Hkv*N*d > 8 Mi elements
 * for N % 128 == 0; the key split uses what the fixed regions leave of the array); otherwise arguments, options and
 * errors as pasa_attn_fwd_ex.  The device that is current at
 * the call must be the stream's.  The first call on a device looks the array's address up (no allocation, but make
 * it before a capture begins).  All calls on one GPU share the one array: calls that may overlap in time on one GPU
 * (different streams, or different threads) race on it and must be serialised by the caller; the array keeps the
 * previous call's contents, none of which a later call reads. */
#define PASA_STATIC_WORKSPACE_BYTES (33u << 20)
int pasa_attn_fwd_static(const void* q, const void* k, const void* v, void* o,
                         int B, int Hq, int Hkv, int N, int d, int causal, float scale,
                         const pasa_opts* opts, void* stream);

/* The two halves of pasa_attn_fwd_ex as separate calls, for callers that attend to the same keys and
 * values more than once (several query chunks against one K/V): pasa_prepare_kv runs Algorithm 1's
 * pre-processing loop (key shift, Eq. (11)) and re-tiles K' and V into `workspace`;
 * pasa_attn_fwd_prepared runs the main loops of Algorithm 1 against such a workspace.  Both calls must be
 * given the same B, Hkv, N, d, scale and opts (beta, variant); pasa_attn_fwd_prepared does not read k or v.
 * It reads the prepared regions and may write the key-split region at the end of the workspace, so calls that use
 * one workspace must not overlap in time.  Same argument rules, workspace size and error codes as pasa_attn_fwd_ex. */
int pasa_prepare_kv(const void* k, const void* v, int B, int Hkv, int N, int d, float scale,
                    const pasa_opts* opts, void* workspace, size_t workspace_bytes, void* stream);
int pasa_attn_fwd_prepared(const void* q, void* o, int B, int Hq, int Hkv, int N, int d, int causal, float scale,
                           const pasa_opts* opts, void* workspace, size_t workspace_bytes, void* stream);

/* The main loops of Algorithm 1 for a chunk of queries against a prepared workspace of N keys (the problem
 * statement of section 1.1 allows different query and key lengths S1 != S2; the paper does not elaborate).
 * q, o: [B, Hq, Nq, d].  Query row r sits at sequence position row0 + r: with causal != 0 it sees the keys
 * n <= row0 + r (row0 = N - Nq aligns the last query with the last key; positions past N - 1 see all keys);
 * with causal == 0 every row sees all N keys and row0 is ignored.  Covers cross-attention, prefill in chunks and
 * decoding against a cache.  pasa_attn_fwd_prepared(..., N, ...) is the case Nq = N, row0 = 0.  A row's result
 * does not depend on the other rows of its chunk.  Splitting a sequence at multiples of 32 rows gives bit-identical output
 * wherever the calls sweep their keys unsplit -- N <= 2048, or at least 192 workgroups of 256 rows (B * Hq * ceil(Nq / 256)) --
 * for pieces of 32 rows or more and, up to 2048 keys, for the end of a causal sequence whatever its length.  Any other
 * call (decoding steps, pieces that start elsewhere, launches that split their keys, calls with counters) agrees up to rounding: it may run
 * on another kernel or sweep the keys in pieces, which moves the level that P is rounded at.  PASA_EINVAL for
 * Nq <= 0 or row0 < 0; otherwise the rules of pasa_attn_fwd_prepared. */
int pasa_attn_fwd_chunk(const void* q, void* o, int B, int Hq, int Hkv, int Nq, int row0, int N, int d, int causal,
                        float scale, const pasa_opts* opts, void* workspace, size_t workspace_bytes, void* stream);

/* An adaptive start of PASA (the paper's closing section names it as future work and gives no mechanism; this is
 * a simple one).  Pass 1 runs the partially low-precision FlashAttention without any shift (PASA_NAIVE16: raw
 * scores rounded to fp16, section 2.1) into o and counts the raw scores that left the fp16 range: in total in
 * *opts->overflow_s, and per (batch, KV head) in counters of its own inside the workspace.  Pass 2 runs
 * opts->variant (not PASA_NAIVE16) into o, but the workgroups of a (batch, KV head) whose counter is zero return at
 * once -- decided on the device, no host synchronisation.  So the query heads of a (batch, KV head) in which nothing
 * overflowed keep the unshifted result, and those of a (batch, KV head) in which some raw score of some query head
 * overflowed get the PASA result (the shifted keys are shared by the query heads of a KV head, so that is the
 * finest unit).  opts and opts->overflow_s (a DEVICE counter the caller has zeroed; it reports the total) are
 * required, opts->nonfinite_o must be NULL.  Otherwise the rules of pasa_attn_fwd_ex. */
int pasa_attn_fwd_adaptive(const void* q, const void* k, const void* v, void* o,
                           int B, int Hq, int Hkv, int N, int d, int causal, float scale,
                           const pasa_opts* opts, void* workspace, size_t workspace_bytes, void* stream);

/* Key pre-processing alone (Algorithm 1's first loop, Eq. (11)): writes, for every 128-key tile,
 * K'[n, c] = fp16((K[n, c] - beta * mean_tile(K[:, c])) * kscale) to kprime in the plain [B, Hkv, N, d]
 * layout.  The mean and the arithmetic are fp64 and the result is rounded once.  For tests and tools;
 * the attention entry points do this internally in their own tiled layout. */
int pasa_shift_keys(const void* k, void* kprime, int B, int Hkv, int N, int d,
                    double beta, double kscale, void* stream);

/* The same with PASA_SHIFT_MATRIX: K'^T = fp16(K^T M16), M16 the entrywise fp16 rounding of Eq. (10)'s M with
 * alpha = 1/kscale.  N must be a multiple of 128. */
int pasa_shift_keys_matrix(const void* k, void* kprime, int B, int Hkv, int N, int d,
                           double beta, double kscale, void* stream);

/* The same contraction on the matrix core (PASA_SHIFT_MATRIX_MFMA): fp32 accumulation, one rounding to fp16. */
int pasa_shift_keys_matrix_mfma(const void* k, void* kprime, int B, int Hkv, int N, int d,
                                double beta, double kscale, void* stream);

/* The shift of PASA_DIRECT: k0[b, h, t, :] = fp16(beta * mean of key tile t) ([B, Hkv, ceil(N/128), d], DEVICE, written)
 * and K' = fp16((K - k0) * kscale) in the plain layout. */
int pasa_shift_keys_direct(const void* k, void* kprime, void* k0, int B, int Hkv, int N, int d,
                           double beta, double kscale, void* stream);

/* ---- A cache of keys and values in 8 bits, in pages, and attention that reads it ----
 *
 * For servers whose sequences grow token by token and differ in length: S sequences share a pool of `pages` pages of `page`
 * tokens each; table[b][i] is the page in the pool that holds the tokens i * page .. i * page + page - 1 of sequence b (sequences
 * may share pages that neither writes).  A token takes d bytes and a scale for its key and for its value, per KV head; what is
 * held stands for code * scale.  Scales belong to a token and head, so a token that enters changes nothing that is there.  (What is
 * brought into the buffers by other means than pasa_cache_write keeps its rules: scales 2^-109 at least, no NaN among the codes.)
 *
 * Eq. (9) of the paper: a vector taken from every key leaves softmax unchanged.  kshift is such a vector per KV head (the bias
 * of the key projection, or a mean over a prompt): it is taken off before keys are rounded to 8 bits, which then need not cover
 * the bias, and attention and the choice of pages never add it back; pasa_cache_read does.
 *
 * kmean holds the mean of the tokens' (shifted, rounded) keys of every page and head: by Eq. (12) a query's product with it is
 * the pseudo-average of the query's scores over that page, which is what pasa_cache_choose ranks pages by.
 *
 * length[b] counts the tokens of sequence b with the ones of the current step: a call that is given rows takes rows
 * row_start[b] .. row_start[b + 1] - 1 as the last ones of sequence b, so row row_start[b] + t of n_b sits at position
 * length[b] - n_b + t.  A step is: length += n, pasa_cache_write, then pasa_attn_cache (after pasa_cache_choose, where not all
 * keys are wanted).  Sequences without rows (n_b = 0) are left alone, as are rows from row_start[S] on.  A step that is taken back
 * (drafted tokens that were not accepted) is a smaller length at the next call; what was written behind it is overwritten.
 *
 * table, length and row_start are read on the device, so that a captured graph follows them; they are not checked by the host.
 * row_start has to ascend.  The kernels keep to the buffers whatever else they hold: lengths are taken as at most table_width * page
 * and at least 0, row_start as between 0 and R; positions before 0 and pages outside the pool are not there (nothing is written to
 * them, they read as zeros and no row sees them). */
typedef enum {
    PASA_CACHE_I8 = 0,    /* bytes hold value + 128, value = -127 .. 127; scale = largest magnitude / 127 */
    PASA_CACHE_E4M3 = 1   /* OCP 8-bit floats, 4 exponent bits; scale = largest magnitude / 448 */
} pasa_cache_format;

typedef struct {
    void* k;              /* DEVICE [pages][Hkv][page][d] bytes, 16-byte aligned, as v */
    void* v;
    float* kscale;        /* DEVICE [pages][Hkv][page], 16-byte aligned, as vscale */
    float* vscale;
    float* kmean;         /* DEVICE [pages][Hkv][d], 16-byte aligned, or NULL: not kept (pasa_cache_choose needs it) */
    const float* kshift;  /* DEVICE [Hkv][d], 16-byte aligned, or NULL: zero.  Constant over the life of the cache's contents */
    const int* table;     /* DEVICE [S][table_width] */
    const int* length;    /* DEVICE [S] */
    int S, Hkv, d;        /* d = 64 or 128 */
    int page;             /* tokens of a page: 16, 32, 64 or 128 */
    int pages, table_width;   /* table_width * page <= 262144 */
    int format;           /* a pasa_cache_format */
} pasa_cache;

/* Tokens enter the cache.  k, v: rows of [Hkv][d] (fp16 or bf16, see pasa_io_dtype), `row_stride` elements apart (at least
 * Hkv * d, a multiple of 8: slices of a joint projection are taken as they are), 16-byte aligned, R rows in all.  Per token and head:
 * scale = fp32(largest magnitude / 127 or 448), 1 where that magnitude is below 2^-100, and codes the nearest of
 * value / scale (ties to even), exactly.  A token with a value that is not finite gets the scale NaN, and so does whoever sees it.
 * kmean != NULL: the means of the pages that are written to are made again, over all their tokens below length[b].
 * PASA_EINVAL also for R <= 0; PASA_EUNSUPPORTED also for 2^23 or more pages (of all heads) that may be written to. */
int pasa_cache_write(const pasa_cache* cache, const void* k, const void* v, int R, long long row_stride, const int* row_start,
                     int io_dtype, void* stream);

/* Positions first[b] .. first[b] + N - 1 of every sequence (first: DEVICE [S], NULL: zeros) as fp16 or bf16 in k, v:
 * [S, Hkv, N, d], 16-byte aligned, what pasa_prepare_kv takes with B = S: a long chunk of a prompt is attended to that way.  code * scale
 * + kshift, rounded to fp32 and then to the type.  Zeros where a sequence has no such position.  PASA_EUNSUPPORTED also where the
 * stretches of 64 tokens (of all sequences and heads) come to 2^24. */
int pasa_cache_read(const pasa_cache* cache, void* k, void* v, const int* first, int N, int io_dtype, void* stream);

/* For every sequence and KV head the pages that its rows' queries point at: the first `head` and the last `tail` pages always (the
 * first ones where they exceed `count`), and of the others those with the largest pseudo-average, max over the rows of the sequence and the query heads of
 * the KV head of q . kmean, in 64 bits; of equal ones the first; NaN counts as the largest.  q: rows of [Hq][d] as k above.  blocks: DEVICE
 * [S][Hkv][count], the places in the sequence's row of the table, ascending, -1 behind the last.  All pages where there are
 * no more than count; none for a sequence without rows.  One row per sequence (Nq = 1 of a decoding step) makes it a choice per
 * query; rows that are to have choices of their own go in as sequences of one row each.  `tail` should cover the pages that the rows themselves lie in.
 * workspace: DEVICE, 256-byte aligned, pasa_cache_choose_workspace() bytes.  PASA_EINVAL also for count < 1, head or tail < 0;
 * PASA_EUNSUPPORTED also where S * Hkv reaches 2^22, or, with count < table_width, S * Hkv * ceil(table_width / 64) 2^24. */
size_t pasa_cache_choose_workspace(const pasa_cache* cache);
int pasa_cache_choose(const pasa_cache* cache, const void* q, int R, long long row_stride, const int* row_start, int Hq, int* blocks,
                      int count, int head, int tail, int io_dtype, void* workspace, size_t workspace_bytes, void* stream);

/* softmax(scale * Q K^T) V of the rows against the cache: decoding steps, chains and trees of drafted tokens.  q: rows of [Hq][d]
 * as above; o: [R][Hq][d], contiguous, 16-byte aligned, not q.  Query head h reads KV head h / (Hq / Hkv).
 * tree == NULL: a row sees the positions up to its own.  tree: DEVICE [R] words of 64 bits: a row sees the positions before its
 * sequence's first row, and that of the sequence's row t iff bit t of its word is set (its own bit among them, if it is to see
 * itself); rows from the 64th on are seen by none.
 * blocks == NULL: all pages.  blocks: DEVICE [S][Hkv][count] as pasa_cache_choose leaves it: only keys of these pages, of those that
 * the row sees; ascending without repeats, -1 behind the last.
 * Scores, statistics and output are held in fp32, P times the value's scale is rounded to fp16 (all its bits from 2^-21 of the row's
 * largest on; the scales of the values that a row sees are meant to lie within 2^80 of each other, where a token whose value is all
 * zeros and has the scale 1 counts as 2^-60), bf16 queries are converted to fp16
 * as they are loaded.  A row that sees no key, or whose scores (times log2(e), in fp32) are all -inf, is zeros.
 * Meant for rows up to some hundred per sequence; more are correct, but long chunks are faster through pasa_cache_read.
 * workspace: DEVICE, 256-byte aligned, pasa_attn_cache_workspace() bytes (which are enough for fewer rows too); calls that share one
 * must not overlap in time.
 * PASA_EUNSUPPORTED also where the rows' blocks of all heads, up to (R * Hq / Hkv / n + S) * Hkv with n = 16, or 32 where a sequence
 * and KV head have more than 16 rows on average, times 40 more than a table's units of 64 keys come to 2^31. */
size_t pasa_attn_cache_workspace(const pasa_cache* cache, int R, int Hq);
int pasa_attn_cache(const pasa_cache* cache, const void* q, void* o, int R, long long row_stride, const int* row_start, int Hq,
                    float scale, const unsigned long long* tree, const int* blocks, int count, int io_dtype, void* workspace,
                    size_t workspace_bytes, void* stream);

/* Host-only, fp64: solves the optimal accuracy condition beta/(1-beta) = f(beta) (Eq. (16), (20)-(22)) by
 * fixed-point iteration from beta0, for a shifting matrix of size n rounded to format tp
 * (0 = fp16, 1 = bf16).  Returns NaN for invalid arguments. */
double pasa_optimal_beta(double beta0, int n, int tp);

/* Host-only: the practical invariance Inva_1 of Eq. (20) for the given beta. */
double pasa_invariance_rounded(double beta, int n, int tp);

const char* pasa_status_string(int status);
int pasa_version(void);

#ifdef __cplusplus
}
#endif
#endif /* PASA_H */
