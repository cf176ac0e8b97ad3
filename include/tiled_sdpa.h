/*
 * tiled_sdpa.h -- C-ABI of the MI355X (gfx950) tiled scaled-dot-product-attention
 * forward library.
 *
 * The operation is the paper's Eq. 1 (Section 3.1) with no mask,
 *
 *     O = softmax(Q K^T * scale) V        per (batch, head),
 *
 * evaluated blockwise with the online-softmax recurrence of Section 4.1.2
 * (Eqs. 2-4: running row maximum m, normaliser l and accumulator o over streamed
 * K/V tiles, final O_i = o_i / l_i), so the S x S score matrix never exists in
 * memory.  Numerics follow Section 4.1.3: FP16 or BF16 inputs and output, FP32
 * accumulation of the dot products, the softmax statistics and the output.
 * The call surface mirrors the functional API of Section 4.2.1,
 * sdpa(q, k, v, causal, scale) -> o; causal = true is TSDPA_FLAG_CAUSAL of tiled_sdpa_fwd_ex.
 *
 * Beside it: attention over dense and paged caches, of 16 or 8 bits, of trees of drafted tokens, the backward pass; and what a serving or
 * training step does around attention: the trees' masks, a cache's pages and slots, norm and rotation of queries and keys, writing to and
 * reading from a cache of 8 bits.
 *
 * All pointers are DEVICE pointers owned by the caller.  The library allocates
 * and frees nothing, keeps no state besides its kernel table, never
 * synchronises, and is thread-safe.  Work is enqueued on `stream`.
 */
#ifndef TILED_SDPA_H
#define TILED_SDPA_H

#ifdef __cplusplus
extern "C" {
#endif

/* element types (Section 4.1.3) */
enum { TSDPA_F16 = 0, TSDPA_BF16 = 1 };

/* status codes: every entry point returns one of these and never throws or aborts */
enum {
    TSDPA_OK = 0,
    TSDPA_ERR_NULL_PTR = 1,      /* q, k, v or o is NULL while B*H*S > 0                    */
    TSDPA_ERR_BAD_SHAPE = 2,     /* negative B, H or S; B*H*ceil(S/64) overflows int; (S+1024)*D*2 >= 2^30 */
    TSDPA_ERR_BAD_DTYPE = 3,     /* dtype is neither TSDPA_F16 nor TSDPA_BF16               */
    TSDPA_ERR_UNSUPPORTED_D = 4, /* D is not 64, 96, 128 or 160                             */
    TSDPA_ERR_MISALIGNED = 5,    /* a tensor base is not 16-byte aligned / lse not 4-byte   */
    TSDPA_ERR_BAD_TILE = 6,      /* (tile_m, tile_n) neither (256,64) nor in {64,128} x {32,64,128},
                                    tile_n = 128 at D = 160 (four such slots fill the LDS), or a
                                    tile the entry point does not offer                       */
    TSDPA_ERR_BAD_SCALE = 7,     /* scale is +-infinity                                     */
    TSDPA_ERR_LAUNCH = 8,        /* the HIP runtime refused the launch                      */
    TSDPA_ERR_WORKSPACE = 9,     /* tiled_sdpa_fwd_kv with more than one split, tiled_sdpa_bwd: workspace NULL,
                                    not 16-byte aligned, or smaller than the matching *_workspace_bytes reports */
    TSDPA_ERR_BAD_SPLITS = 10,   /* splits < 0 or > TSDPA_MAX_SPLITS                         */
    TSDPA_ERR_STATIC_SCRATCH = 11, /* tiled_sdpa_fwd_kvcache_static: the split states need more than
                                    TSDPA_STATIC_SCRATCH_BYTES, or the buffer's address cannot be obtained */
    TSDPA_ERR_BAD_EPS = 12,      /* eps is negative, infinite or NaN                         */
    TSDPA_ERR_BAD_STRIDE = 13    /* a stride of rows is negative or not a multiple of 8 elements, or rows to be written overlap */
};

enum { TSDPA_MAX_SPLITS = 128 };
enum { TSDPA_TUNE_TILES = 7 };      /* candidates of tiled_sdpa_tune_tile */

/* size of the library-owned device buffer behind tiled_sdpa_fwd_kvcache_static (32 MiB per GPU) */
enum { TSDPA_STATIC_SCRATCH_BYTES = 32 * 1024 * 1024 };

/* flags for tiled_sdpa_fwd_ex */
enum {
    TSDPA_FLAG_LINEAR_GRID = 1u, /* workgroup i handles tile i (no per-XCD regrouping); for measurements */
    TSDPA_FLAG_EXACT_MAX = 2u,   /* raise the softmax reference m on every new row maximum (Eq. 2 literally).
                                    Default: the weights of a tile are taken against the current reference
                                    first, and it is raised (to the tile maximum, with the rescale of
                                    Eqs. 3-4) only when their sum exceeds 2^8; this gives the same O and lse
                                    up to rounding and spares most tiles the maximum and the rescale.  With
                                    the flag most tiles are computed twice: for checking, not for speed. */
    TSDPA_FLAG_CAUSAL = 8u       /* causal mask (Section 4.1.3; Eq. 1 with M_ij = -inf for j > i): key j
                                    contributes to query row i only if j <= i.  K/V tiles strictly above
                                    the diagonal of a workgroup's rows are neither read nor computed. */
};

/*
 * Forward pass, Eq. 1 via Eqs. 2-4.
 *
 *   q, k, v : [B, H, S, D] contiguous row-major, element type `dtype`, device memory,
 *             16-byte aligned (Section 4.1.1 layout; viewed as [B*H, S, D] and tiled along S).
 *   o       : [B, H, S, D], same type; every element is overwritten.  Must not alias q, k, v.
 *   lse     : optional (NULL to skip) FP32 [B, H, S]; receives m_i + ln(l_i), the natural-log
 *             normaliser of row i, which is what merging partial results over key ranges needs.
 *   S       : any length >= 0; key columns beyond S contribute nothing and rows beyond S are
 *             neither computed into memory nor read past the tensor end.
 *   D       : 64, 96, 128 or 160 (the head dims of the paper's grid, Section 4.3).
 *   scale   : multiplies Q K^T; any finite value.  NaN selects the default 1/sqrt(D)
 *             (Section 4.2.1), since C has no default arguments.
 *   stream  : hipStream_t (NULL = default stream).  The call returns once the kernel is enqueued.
 *
 * Validation order: dtype, D, shape, empty problem (B*H*S == 0 returns TSDPA_OK without
 * touching memory), null pointers, alignment, tile, scale, launch.
 */
int tiled_sdpa_fwd(const void *q, const void *k, const void *v, void *o, float *lse,
                   int B, int H, int S, int D, float scale, int dtype, void *stream);

/*
 * Same operation with the schedule exposed (Table 1 of the paper: T_M query rows per
 * workgroup, T_N key/value rows per streamed tile).  tile_m in {64,128}, tile_n in
 * {32,64,128} (128 not at D = 160), or (tile_m, tile_n) = (256, 64), which is not in the paper's grid: eight
 * wavefronts share every K/V tile, the fastest schedule on this GPU for long sequences at D >= 96 without the
 * causal mask.
 * tile_m = tile_n = 0 selects the built-in shape heuristic, which is what tiled_sdpa_fwd uses; where workgroups would be
 * few it also splits the key tiles over several streams inside a workgroup, which explicit tiles never do.  The
 * result does not depend on the tile choice beyond rounding order.
 */
int tiled_sdpa_fwd_ex(const void *q, const void *k, const void *v, void *o, float *lse,
                      int B, int H, int S, int D, float scale, int dtype, void *stream,
                      int tile_m, int tile_n, unsigned flags);

/* The (tile_m, tile_n) the heuristic picks for a shape and flags (only TSDPA_FLAG_CAUSAL matters), that of the form
 * without streams; returns a status code. */
int tiled_sdpa_default_tile(int B, int H, int S, int D, int dtype, unsigned flags, int *tile_m, int *tile_n);

/*
 * Schedule search (the tuning policy of Table 1 and Sections 5.5-5.6: a small set of tile candidates, the
 * best one kept per problem shape): runs the forward pass of tiled_sdpa_fwd_ex with every legal
 * (tile_m, tile_n) on the caller's tensors -- one untimed launch, then `launches` (1..1000) timed
 * ones between two HIP events on `stream` -- and reports the fastest in *tile_m, *tile_n.  Unlike
 * every other entry point this one WAITS for the stream (once per candidate); it keeps no record, the
 * caller passes the result to tiled_sdpa_fwd_ex.  o is overwritten (with the correct result).
 * ms_per_launch: NULL, or host array of TSDPA_TUNE_TILES (7) floats that receives the time per launch of
 * (64,32) (64,64) (64,128) (128,32) (128,64) (128,128) (256,64) in that order, -1 for a tile that is not
 * offered at this D.  An empty problem returns the heuristic's tile and measures nothing.
 * The candidates are the explicit tiles: the streams that tile_m = tile_n = 0 takes where workgroups are few (up to 400 of
 * 128 query rows) are none of them, and there 0, 0 is up to three times as fast as the best tile reported here.
 * Validation as tiled_sdpa_fwd_ex; launches out of range is TSDPA_ERR_BAD_SHAPE; tile_m or tile_n
 * NULL is TSDPA_ERR_NULL_PTR.  Timings are only meaningful on an otherwise idle GPU (Section 4.2.3).
 */
int tiled_sdpa_tune_tile(const void *q, const void *k, const void *v, void *o,
                         int B, int H, int S, int D, float scale, int dtype, void *stream, unsigned flags,
                         int launches, int *tile_m, int *tile_n, float *ms_per_launch);

/*
 * Forward pass for Sq query rows against Skv key/value rows, with the key range optionally split
 * over several workgroups: the KV-cache / decoding shapes that the paper names as future work
 * (Section 7), and the cure for shapes whose B*H*ceil(Sq/tile_m) workgroups cannot fill the GPU.
 * Each split runs the recurrence of Section 4.1.2 (Eqs. 2-4) over its own contiguous run of K/V
 * tiles and leaves its state (o, m, l) in the workspace; a second kernel (or, on a decoding step with few
 * states per head, the workgroup that finishes last; o then holds its marks until the result replaces them)
 * combines the states with the rescaling of Eqs. 3-4 and applies the final O_i = o_i / l_i.
 *
 *   q        : [B, H, Sq, D];  k, v : [B, H, Skv, D];  o : [B, H, Sq, D];  lse : NULL or FP32 [B, H, Sq].
 *              Layout, alignment, D, scale, dtype, stream as for tiled_sdpa_fwd.
 *   flags    : TSDPA_FLAG_CAUSAL takes the Sq queries to be the LAST Sq positions of the Skv-long
 *              sequence (the paper defines the mask for Sq = Skv only): key j contributes to query
 *              row i only if j <= i + Skv - Sq.  It needs Skv >= Sq.  The other flags as above.
 *   tile_m   : 64 or 128;  tile_n : 32 or 64;  or (256, 64) (not with a paged cache);  both 0 = heuristic.
 *   splits   : workgroups per (head, query tile) along the key axis, 1..TSDPA_MAX_SPLITS; 0 = the
 *              value tiled_sdpa_kv_default_splits reports for this shape and these flags, or with an explicit
 *              tile the value of tiled_sdpa_kv_tile_splits where the workspace is large enough for it.
 *   workspace: device memory for the split states, 16-byte aligned, at least
 *              tiled_sdpa_kv_workspace_bytes(B, H, Sq, D, n) bytes, n being `splits` or, for splits = 0,
 *              the heuristic's value; ignored (may be NULL) when n = 1, where O is written directly.
 *              Owned by the caller; the library uses it only inside this call's kernels, so
 *              calls that may overlap on the GPU need distinct workspaces.  Its contents afterwards
 *              are unspecified.  More splits than there are K/V tiles are allowed (the surplus ones
 *              contribute nothing) but waste workspace.
 *
 * Skv = 0 with Sq > 0 is TSDPA_ERR_BAD_SHAPE (a softmax over no keys).  Validation order: dtype, D,
 * shape, empty problem (B*H*Sq == 0), null pointers, alignment, tile, scale, splits, workspace, launch.
 */
int tiled_sdpa_fwd_kv(const void *q, const void *k, const void *v, void *o, float *lse,
                      int B, int H, int Sq, int Skv, int D, float scale, int dtype, void *stream,
                      int tile_m, int tile_n, unsigned flags,
                      int splits, void *workspace, unsigned long long workspace_bytes);

/*
 * tiled_sdpa_fwd_kv with grouped heads: H query heads read Hkv key/value heads, query head h the
 * key/value head h / (H / Hkv) -- the layout of multi-query and grouped-query KV caches.  The paper
 * has one key/value head per query head (Section 3.1); per query head this computes the same Eq. 1,
 * with the causal limit of tiled_sdpa_fwd_kv for each head's Sq rows.
 *
 *   q, o : [B, H, Sq, D];  lse : NULL or FP32 [B, H, Sq];  k, v : [B, Hkv, Skv, D];  H % Hkv == 0.
 *   Everything else as for tiled_sdpa_fwd_kv, which is this call with Hkv = H.  The heuristics see
 *   B * Hkv heads of (H / Hkv) * Sq rows each: tiled_sdpa_kv_default_splits(B, Hkv, (H / Hkv) * Sq, ...)
 *   without the causal flag reports the split count used for splits = 0, and the workspace size is
 *   tiled_sdpa_kv_workspace_bytes(B, H, Sq, D, n).
 *
 * The query heads of a group are adjacent in memory, so a group's (H / Hkv) * Sq rows form one run of
 * rows that streams the group's keys and values once (instead of once per query head): on a
 * decoding step the otherwise empty rows of the 32-row MFMA tile carry the other heads of the
 * group.  Hkv <= 0 with H > 0, or H not a multiple of Hkv, is TSDPA_ERR_BAD_SHAPE (checked right
 * after the shape checks of tiled_sdpa_fwd_kv).
 */
int tiled_sdpa_fwd_gqa(const void *q, const void *k, const void *v, void *o, float *lse,
                       int B, int H, int Hkv, int Sq, int Skv, int D, float scale, int dtype, void *stream,
                       int tile_m, int tile_n, unsigned flags,
                       int splits, void *workspace, unsigned long long workspace_bytes);

/*
 * tiled_sdpa_fwd_gqa over a KV cache whose batch entries are filled to different lengths (the
 * serving form of the KV-cache variants the paper names as future work, Section 7): k and v are
 * [B, Hkv, Skv, D] with Skv the CAPACITY of the cache, and batch entry b holds kv_lens[b] valid key
 * rows at the front of each of its heads.
 *
 *   kv_lens : device pointer to B 32-bit integers, 4-byte aligned, read by the kernels when they run
 *             (not by this call); values are clamped to [0, Skv].  NULL = every entry holds Skv rows,
 *             which is tiled_sdpa_fwd_gqa.
 *
 * Entry b is computed as tiled_sdpa_fwd_gqa would compute it on its first kv_lens[b] key rows: rows
 * past the length are never fetched, and under TSDPA_FLAG_CAUSAL the Sq queries are the last Sq
 * positions of the kv_lens[b]-long sequence (key j contributes to query row i only if
 * j <= i + kv_lens[b] - Sq).  A query row that no key reaches -- an empty entry, or under the causal
 * flag an entry shorter than Sq for its first Sq - kv_lens[b] rows -- gets O = 0 and LSE = -infinity
 * (a softmax over no keys has no value; zero is what leaves a residual stream untouched).  A row with a score that is
 * NaN has O = LSE = NaN, whatever the number of splits.  Shapes are
 * validated against the capacity; the split heuristic sees the capacity too, so workspace sizes do not
 * depend on the lengths.  Everything else as for tiled_sdpa_fwd_gqa.
 */
int tiled_sdpa_fwd_kvcache(const void *q, const void *k, const void *v, void *o, float *lse, const int *kv_lens,
                           int B, int H, int Hkv, int Sq, int Skv, int D, float scale, int dtype, void *stream,
                           int tile_m, int tile_n, unsigned flags,
                           int splits, void *workspace, unsigned long long workspace_bytes);

/*
 * tiled_sdpa_fwd_kvcache for callers that cannot allocate device memory and so have no workspace to
 * pass: code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  The split
 * states go to a buffer of TSDPA_STATIC_SCRATCH_BYTES that is part of the library's device code (a
 * file-scope __device__ array: every GPU the library runs on holds its own copy from the first use of
 * the library on it until the process ends).  The call itself allocates and frees nothing and does not
 * synchronise; the first call on a device looks the buffer's address up once.
 *
 *   All arguments as for tiled_sdpa_fwd_kvcache (kv_lens NULL = a full cache, Hkv = H = plain heads),
 *   minus the workspace.  Results are bit-identical to tiled_sdpa_fwd_kvcache with the same tile and
 *   split count: the same kernels run.
 *   Limit: tiled_sdpa_kv_workspace_bytes(B, H, Sq, D, n) <= TSDPA_STATIC_SCRATCH_BYTES, n being `splits`
 *   or the heuristic's count for splits = 0 (which is smaller here where the default count does not fit); beyond it the call enqueues nothing and returns
 *   TSDPA_ERR_STATIC_SCRATCH (pass fewer splits, or use tiled_sdpa_fwd_kvcache).  n = 1 needs no scratch.
 *   Nothing in the buffer has to start at zero: every word the second kernel reads is written by the
 *   first kernel of the same call; its contents after a call are unspecified.
 *   ALL calls on one GPU share that GPU's buffer: calls that may overlap on the GPU (different streams,
 *   or graphs replayed concurrently) race on it and must be serialised by the caller; calls on one
 *   stream are ordered and safe.
 *
 * Validation order: dtype, D, shape, empty problem, splits, tile (when the heuristic split count needs
 * it), static-scratch size, then everything tiled_sdpa_fwd_kvcache checks.
 */
int tiled_sdpa_fwd_kvcache_static(const void *q, const void *k, const void *v, void *o, float *lse,
                                  const int *kv_lens, int B, int H, int Hkv, int Sq, int Skv, int D, float scale,
                                  int dtype, void *stream, int tile_m, int tile_n, unsigned flags, int splits);

/*
 * tiled_sdpa_fwd_kvcache over a PAGED cache (the KV-cache variants of the paper's roadmap, Section 7,
 * in the form serving systems store them): keys and values live in pages of block_rows rows that any
 * batch entry may own in any order.
 *
 *   k_pages, v_pages : [P, Hkv, block_rows, D], P pages (P is not passed: the table names the pages);
 *                      16-byte aligned.  block_rows is 64, 128, 256, ... (a power of two >= 64, so that a
 *                      K/V tile of 32 or 64 rows lies within one page).
 *   block_table      : device, int32 [B, max_blocks], 4-byte aligned: block_table[b][i] is the page
 *                      holding key rows i*block_rows ... (i+1)*block_rows - 1 of batch entry b.  Only
 *                      the entries below ceil(kv_lens[b] / block_rows) are used; the others may hold
 *                      anything.  The pages named must exist; the library cannot check that.
 *   kv_lens          : device, int32 [B]: valid key rows of entry b, clamped to
 *                      [0, max_blocks * block_rows].  Required (not NULL).
 *   q, o, lse, H, Hkv, Sq, D, scale, dtype, stream, tiles, flags, splits, workspace: as for
 *                      tiled_sdpa_fwd_kvcache with capacity Skv = max_blocks * block_rows (that is
 *                      what shapes are validated against and what the split heuristic sees).
 *
 * Both arrays are read by the kernels when they run.  Every K/V tile is fetched through a buffer
 * descriptor of its own that starts at the tile's rows within its page and is as long as the tile has
 * valid rows, so neither rows past kv_lens[b] nor pages past the last one are touched.  Results are
 * those of tiled_sdpa_fwd_kvcache on the same rows gathered into a dense cache.  block_rows not a
 * power of two >= 64, max_blocks < 0 or max_blocks * block_rows overflowing an int is
 * TSDPA_ERR_BAD_SHAPE; kv_lens or block_table NULL with B*H*Sq > 0 is TSDPA_ERR_NULL_PTR.
 */
int tiled_sdpa_fwd_paged(const void *q, const void *k_pages, const void *v_pages, void *o, float *lse,
                         const int *kv_lens, const int *block_table,
                         int B, int H, int Hkv, int Sq, int max_blocks, int block_rows, int D,
                         float scale, int dtype, void *stream, int tile_m, int tile_n, unsigned flags,
                         int splits, void *workspace, unsigned long long workspace_bytes);

/*
 * tiled_sdpa_fwd_kvcache and tiled_sdpa_fwd_paged for a tree of drafted tokens (speculative decoding): the T queries of an entry are
 * tokens of a tree whose keys are the last T rows of the entry's kv_lens[b], and each sees the rows before those (the cached
 * sequence) and the tokens that its mask names.
 *
 *   mask       : device int64, ceil(T / 64) words per token, 8-byte aligned: bit j % 64 of word j / 64 of token i is set iff token i sees
 *                token j (key row kv_lens[b] - T + j); tiled_sdpa_tree_mask makes it, any other pattern is as good.  Bits from T on are
 *                not looked at, nor are those of rows before the entry's first (an entry shorter than T).
 *   mask_batch : words from one entry's mask to the next (at least T * ceil(T / 64)), 0 = one mask for all entries.
 *
 * A token that sees no key gets O = 0 and LSE = -infinity.  Values of keys that a token does not see do not reach it, whatever they
 * are: rows of k or v of other tokens may hold infinities and NaN.  T <= 65536; everything else as for the two calls named
 * (the tile is the library's choice).  With splits = 0 and a workspace of tiled_sdpa_kv_workspace_bytes(B, H, T, D, n), n being what
 * tiled_sdpa_tree_default_splits reports (Skv: the capacity), the call takes the form that runs best; with less, what runs best in that.
 */
int tiled_sdpa_fwd_tree(const void *q, const void *k, const void *v, void *o, float *lse, const int *kv_lens,
                        const long long *mask, long long mask_batch, int B, int H, int Hkv, int T, int Skv, int D,
                        float scale, int dtype, void *stream, int splits, void *workspace, unsigned long long workspace_bytes);
int tiled_sdpa_fwd_tree_paged(const void *q, const void *k_pages, const void *v_pages, void *o, float *lse,
                              const int *kv_lens, const int *block_table, const long long *mask, long long mask_batch,
                              int B, int H, int Hkv, int T, int max_blocks, int block_rows, int D,
                              float scale, int dtype, void *stream, int splits, void *workspace, unsigned long long workspace_bytes);

int tiled_sdpa_tree_default_splits(int B, int H, int Hkv, int T, int Skv, int D, int dtype, int *splits);

/* Splits the heuristic picks (1 when the query tiles alone fill the GPU); returns a status code. */
int tiled_sdpa_kv_default_splits(int B, int H, int Sq, int Skv, int D, int dtype, unsigned flags, int *splits);
/* The same for a call with an explicit tile (both 0: the value above).  The two differ where the heuristic would
 * take the decoding kernel or streams, which explicit tiles never do.  TSDPA_ERR_BAD_TILE for a tile the cache entry points
 * do not offer. */
int tiled_sdpa_kv_tile_splits(int B, int H, int Sq, int Skv, int D, int dtype, unsigned flags, int tile_m, int tile_n, int *splits);

/* Workspace bytes tiled_sdpa_fwd_kv needs for `splits` >= 1 (a value from tiled_sdpa_kv_default_splits,
 * or the caller's own): B*H*splits*Sq*(D+2) floats.  0 for splits <= 1 or negative arguments.
 * The counts above are at most 2048 workgroups of 128 rows (170 MB at D = 160), and, but for 33 to 64 rows per key/value head,
 * never fewer for a longer cache: a workspace sized for the capacity serves every shorter length with splits = 0.  Where a call with
 * splits = 0 is given less, it takes a smaller count (512 workgroups in all, rounded up) if that fits. */
unsigned long long tiled_sdpa_kv_workspace_bytes(int B, int H, int Sq, int D, int splits);

/*
 * Backward pass: gradients of a scalar loss with respect to q, k and v, given dout = d(loss)/d(o).
 * The paper leaves the backward pass as future work (Section 7); this is the derivative of its
 * Eq. 1 (Section 3.1), evaluated tile by tile with the probabilities recomputed from the forward
 * pass's log-sum-exp (never stored), in FP32 with 16-bit MFMA operands as in Section 4.1.3:
 *     P = exp(scale * Q K^T [+ causal mask] - lse),  dV = P^T dO,  dP = dO V^T,
 *     dS = P * (dP - rowsum(dO * O)),  dQ = scale * dS K,  dK = scale * dS^T Q.
 *
 *   q, k, v, o, dout : [B, H, S, D] as for tiled_sdpa_fwd; o and lse are that call's outputs for the
 *                      same q, k, v, scale and flags (lse is required here).
 *   dq, dk, dv       : [B, H, S, D], same type; every element is overwritten.  Must not alias inputs.
 *   flags            : TSDPA_FLAG_CAUSAL or 0.
 *   workspace        : device memory, 16-byte aligned, at least tiled_sdpa_bwd_workspace_bytes(B, H, S)
 *                      bytes (two FP32 values per query row); caller-owned, used only during this call's
 *                      kernels, so calls that may overlap on the GPU need distinct workspaces.  With
 *                      tiled_sdpa_bwd_full_workspace_bytes bytes or more a large call takes five products
 *                      instead of seven (0.9 of the time on average).
 * Kernels enqueued on `stream`: dQ, which also leaves the row statistics in the workspace, or a kernel for these alone (Delta_i = <dO_i, O_i> and
 * LSE_i in log2 units; for query rows that see at most 64 keys -- S <= 64, or the first 64 rows under the causal mask --
 * Delta_i by its definition sum_j P_ij dP_ij in FP32, because on such rows the rounding of the 16-bit o inside
 * <dO_i, O_i> is not attenuated by small P_ij); then dK and dV in one pass over resident keys, in one grid with dQ where
 * that was not computed before.  Sequences of up to 256 rows
 * at D = 64 and 96 with H = Hkv may take one kernel for all of it, which leaves the workspace alone.  No sum crosses
 * workgroups there.  With the full workspace, a kernel for the statistics and one for all three gradients, in which the parts of a
 * query row's dQ are summed across workgroups in a fixed order.  Results are deterministic either way, and depend on
 * workspace_bytes only by which of the two it is: their orders of summation differ in the last bits.
 * Values that are not finite: under the causal mask a row of q (with its o and lse) or dout that holds one may make NaN of dk and dv of keys that
 * it does not see, up to 127 rows behind it (full workspace: to the end of its 32 rows, counted from row 0), and a row of k of the dq of
 * as many rows before it.  Validation order: dtype, D, shape, empty problem, null pointers, alignment,
 * scale, workspace, launch.
 */
int tiled_sdpa_bwd(const void *q, const void *k, const void *v, const void *o, const void *dout,
                   const float *lse, void *dq, void *dk, void *dv,
                   int B, int H, int S, int D, float scale, int dtype, unsigned flags,
                   void *workspace, unsigned long long workspace_bytes, void *stream);

/*
 * tiled_sdpa_bwd with grouped heads (the backward pass of tiled_sdpa_fwd_gqa at Sq = Skv = S): H query
 * heads read Hkv key/value heads, query head h the head h / (H / Hkv).  q, o, dout, dq : [B, H, S, D];
 * lse : [B, H, S];  k, v, dk, dv : [B, Hkv, S, D].  dq is the gradient of each query head against the
 * keys and values of its group; dk and dv are the gradients summed over the query heads of the group
 * (the chain rule of sharing one head among them), accumulated in FP32 inside one workgroup per
 * (key/value head, key tile), in a fixed order: results are deterministic.  Workspace as for
 * tiled_sdpa_bwd(B, H, S).  Everything else, validation included, as tiled_sdpa_bwd, which is this call
 * with Hkv = H; Hkv <= 0 with H > 0 or H not a multiple of Hkv is TSDPA_ERR_BAD_SHAPE.
 */
int tiled_sdpa_bwd_gqa(const void *q, const void *k, const void *v, const void *o, const void *dout,
                       const float *lse, void *dq, void *dk, void *dv,
                       int B, int H, int Hkv, int S, int D, float scale, int dtype, unsigned flags,
                       void *workspace, unsigned long long workspace_bytes, void *stream);

/* Workspace bytes tiled_sdpa_bwd needs: 2 * (B*H*S + 128) floats.  0 for negative arguments. */
unsigned long long tiled_sdpa_bwd_workspace_bytes(int B, int H, int S);

/* Workspace bytes with which tiled_sdpa_bwd (Hkv = H) and tiled_sdpa_bwd_gqa are fastest: for large problems at D = 64, 96 and 128 room for
 * FP32 sums of dQ, about 4*B*H*S*D bytes and at most 2.3 GB; otherwise what tiled_sdpa_bwd_workspace_bytes says.  flags as for the
 * call.  Never fails: for arguments that the call refuses, the latter too. */
unsigned long long tiled_sdpa_bwd_full_workspace_bytes(int B, int H, int Hkv, int S, int D, unsigned flags);

/*
 * ---- Around attention: trees of drafted tokens, a cache's pages, and queries and keys on their way to attention.
 *
 * Trees of drafted tokens (speculative decoding): parents [B, T] -> which tokens each token follows.
 *
 *   parents : device int32 [B, T]: the token that token i of a tree follows, an earlier one (0 <= parent < i); any other value
 *             means that i follows the cached sequence itself.
 *   mask    : device int64 [B, T, ceil(T/64)]: bit j % 64 of word j / 64 of row i is set iff j is i or one of its ancestors: what
 *             tiled_sdpa_fwd_tree reads.  One mask serves all layers of a step.
 *   depths  : NULL, or device int32 [B, T]: the number of ancestors: the token's distance from the first position behind the
 *             cached sequence (see tiled_sdpa_cache_step).
 *   T       : 0 ... 1024.
 * In a batch of trees of several sizes a tree of n < T tokens takes the last n places, behind a chain (token i follows i - 1) of T - n
 * that its first tokens follow: the chain stands for the last T - n rows of the cached sequence, which all tokens see.
 * The outputs must not overlap parents.
 */
int tiled_sdpa_tree_mask(const int *parents, long long *mask, int *depths, int B, int T, void *stream);

/*
 * The cache's side of a serving step: every entry of a batch appends tokens or drops some, and gets the pages it needs for
 * that, the slot of each new token, and its position.  Nothing is read back by the host: a captured step serves any lengths.
 *
 *   kv_lens      : device int32 [B]: rows of each entry now.  An entry holds exactly ceil(rows / block_rows) pages, the first of
 *                  its row of block_table.
 *   counts       : device int32 [B]: rows to append (0 ... S), or to drop (negative; -kv_lens[b] for a request that is done).  What is
 *                  dropped are an entry's LAST rows, whichever tokens they hold: of drafts in a chain the rejected ones.  The accepted
 *                  tokens of a tree that branches are a path through it, in general not the first of its rows: the caller moves
 *                  their rows of K and V to the front of the tree's first (row i of the tree to slot i of those that this call
 *                  returned; a token's position, that of its depth, is then its row's), or siblings' rows stay in their place.
 *   depths       : NULL, or device int32 [B, S] (tiled_sdpa_tree_mask): token i of an entry has position
 *                  new_lens[b] - S + depths[b][i] instead of the one of its row.
 *   block_table  : device int32 [B, max_blocks], in and out: as for tiled_sdpa_fwd_paged.  NULL = a dense cache [B, Hkv, block_rows, D]
 *                  (entry b's rows are slots b * block_rows ...); free_pages and pool are then not looked at.
 *   free_pages   : device int32 [pool_size], in and out: pages that no entry holds, the first pool[0] of them; room for all pages
 *                  (page numbers are below pool_size).
 *   pool         : device int32 [2]; pool[0] = pages in free_pages.
 *   new_lens     : device int32 [B]: kv_lens + counts.
 *   slots        : device int32 [B, S]: row new_lens[b] - S + i of entry b for token i, as page * block_rows + row in the page, if the
 *                  step appended it; else -1 (entries with fewer than S new tokens have them at the end, as the queries of
 *                  TSDPA_FLAG_CAUSAL are the last positions).
 *   positions    : device int32 [B, S]: the row's position (0 where there is no slot).
 *   new_pool     : device int32 [2]: pages free after the step, and 0; or, of a step that is REFUSED, the pages as they were and
 *                  what is missing: pages (dense: rows) that the pool or the ends of entries lack (of one entry's end at most 65536
 *                  are counted), -1 if a length, count or pool cannot be one (negative, beyond the capacity, more than S).  A refused step changes nothing: new_lens =
 *                  kv_lens, every slot -1.
 *
 * Pages go in this order: those given up (entry by entry) to those needed (entry by entry), then from the end of the pool; what is
 * left of those given up goes on its end, the first last, so that dropping what was appended restores the pool.  Only
 * block_table's columns from the pages held on and free_pages' elements from pool[0] on are written.  The outputs must not
 * overlap the inputs (new_lens and new_pool are others than kv_lens and pool, to be exchanged from step to step).
 * B <= 8192; page numbers times block_rows, B * S and B * max_blocks fit an int.
 */
int tiled_sdpa_cache_step(const int *kv_lens, const int *counts, const int *depths, int *block_table, int *free_pages, const int *pool,
                          int *new_lens, int *slots, int *positions, int *new_pool,
                          int B, int S, int max_blocks, int block_rows, int pool_size, void *stream);

/* Rows of D values of [B, S, heads, D], strides in elements: a projection's output, or a view into a packed one.  data is 16-byte
 * aligned, the values of a row are adjacent, the strides are multiples of 8 (that of a dimension of one or none is not looked at). */
typedef struct {
    void *data;
    long long batch, row, head;
} tsdpa_rows;

enum { TSDPA_FLAG_INTERLEAVED = 16u };   /* pairs are neighbouring columns (2 i, 2 i + 1) instead of (i, i + rot / 2) */
enum { TSDPA_F32 = 2 };                  /* a type of weights */

/* Norm and rotation of queries and keys: what the three calls below have in common. */
typedef struct {
    int B, S, H, Hkv, D;         /* D: 64, 96, 128 or 160 */
    int dtype;                   /* of the rows: TSDPA_F16 or TSDPA_BF16 */
    int rot;                     /* columns 0 ... rot - 1 are rotated; a multiple of 16, 0 ... D */
    unsigned flags;              /* TSDPA_FLAG_INTERLEAVED or 0 */
    float eps;                   /* >= 0 */
    int weight_dtype;            /* TSDPA_F32 or the rows' */
    const void *q_weight, *k_weight;   /* device [D], 16-byte aligned; NULL: that tensor is rotated without a norm */
    const int *positions;        /* device int32; token (b, s) is at positions[axis * pos_axis + b * pos_batch + s] on an axis */
    long long pos_batch, pos_axis;
    const float *inv_freq;       /* device FP32 [rot / 2]: angle of a pair = position * inv_freq, radians */
    const int *axes;             /* NULL (one axis), or device int32 [rot / 2]: the axis of each pair, 0 ... n_axes - 1 (clamped to that) */
    int n_axes;
} tsdpa_rope;

/*
 * Queries and keys from the projection to attention, in one pass: the RMS norm of each head's row, the weight of each column, the
 * rotation of each pair (a, b) by its angle,
 *     y = x / sqrt(mean(x^2) + eps) * w,     (y_a cos - y_b sin, y_b cos + y_a sin),
 * and the layout.  FP32 throughout (angles in 64 bits up to whole turns: any position is as exact as the first), one rounding.  The mean
 * of squares is taken in FP32: rows of BF16 values whose squares overflow it (beyond 1e18) have no norm, nor, with eps = 0, rows
 * whose squares all fall below it (1e-19); an eps below 1.2e-38 (FP32's smallest normal number) counts as 0.  Columns from rot on
 * are only normed and weighted: what another column holds, infinities and NaN included, reaches them through the row's mean alone.
 *
 *   q, k         : tsdpa_rows of [B, S, H, D] and [B, S, Hkv, D].
 *   q_out, k_out : [B, H, S, D] and [B, Hkv, S, D], contiguous, 16-byte aligned: what tiled_sdpa_fwd and its kin read.  Must overlap
 *                  neither each other nor the inputs.
 *
 * Validation order, of all three calls: dtypes, D, shape (rot, n_axes, the cache's among it), empty problem, null pointers, alignment,
 * strides, eps, workspace, launch.
 */
int tiled_sdpa_qk_norm_rope(const tsdpa_rope *p, const tsdpa_rows *q, const tsdpa_rows *k, void *q_out, void *k_out, void *stream);

/*
 * The serving form: q as above, k (normed, rotated) and v (as it is) to their slots of a cache.
 *
 *   v                : tsdpa_rows of [B, S, Hkv, D].
 *   slots            : device int32 [B, S] (tiled_sdpa_cache_step): token's row in the cache, page * block_rows + row in the page.  A
 *                      token whose slot is negative or past the last page's is not written.  Tokens with the same slot: one of them
 *                      is, row by row and which one is not said.
 *   k_cache, v_cache : [pages, Hkv, block_rows, D] (of a dense cache [B, Hkv, Skv, D]: pages = B, block_rows = Skv); pages *
 *                      block_rows fits an int.  Other rows are left as they are.  q_out and the caches must overlap neither each
 *                      other nor the inputs (rows that another token's part of the call still reads, among them).
 */
int tiled_sdpa_qk_norm_rope_cache(const tsdpa_rope *p, const tsdpa_rows *q, const tsdpa_rows *k, const tsdpa_rows *v, const int *slots,
                                  void *q_out, void *k_cache, void *v_cache, int pages, int block_rows, void *stream);

/*
 * Backward of tiled_sdpa_qk_norm_rope: given the gradients of q_out and k_out, those of q, k and the weights.  With g the gradient
 * rotated back and r = 1 / sqrt(mean(x^2) + eps) (computed again):
 *     dw = sum over the rows of g * x * r,     dx = r * (g * w - x * r * mean(g * w * x * r)).
 *
 *   dq_out, dk_out     : [B, H, S, D] and [B, Hkv, S, D], contiguous, 16-byte aligned.
 *   q, k               : as for the forward call (without weights they are not looked at).
 *   dq, dk             : tsdpa_rows to be written, of the shapes of q and k; every element is overwritten.  Must overlap neither each
 *                        other (views of one packed tensor that share no element do not) nor the inputs that are looked at.
 *   dq_weight, dk_weight : [D] in weight_dtype; not looked at (may be NULL) where there is no weight.
 *   workspace          : device, 16-byte aligned, at least tiled_sdpa_qk_norm_rope_bwd_workspace_bytes(B, S, D) bytes; not looked at
 *                        without weights.  Calls that may overlap on the GPU need distinct ones.
 * The weights' sums are FP32 in a fixed order: results are deterministic.
 */
int tiled_sdpa_qk_norm_rope_bwd(const tsdpa_rope *p, const void *dq_out, const void *dk_out, const tsdpa_rows *q, const tsdpa_rows *k,
                                const tsdpa_rows *dq, const tsdpa_rows *dk, void *dq_weight, void *dk_weight,
                                void *workspace, unsigned long long workspace_bytes, void *stream);
unsigned long long tiled_sdpa_qk_norm_rope_bwd_workspace_bytes(int B, int S, int D);

/*
 * ---- A cache of 8 bits: half the bytes of a 16-bit one to read in a decoding step, and to hold.
 *
 * A value is code * 2^E.  Codes are E4M3 (sign, four bits of exponent, three of mantissa; largest 448; 0x7f and 0xff are NaN, there is no
 * infinity); 32 consecutive rows (0 ... 31, 32 ... 63, ... of an entry) of a head of K share one E, and of V another, kept as the byte
 * E + 127, -62 <= E <= 62 (other bytes count as the nearest of these).  A power of two, because the codes are floating point themselves: a
 * finer scale would gain the top of their range at most, and products with this one are exact.  What is stored is within 2^-4 of a value,
 * or, where that is less, within 2^-10 * 2^E (2^-9 * 2^E in rows that were there when the scale grew), and E is the least with which the largest
 * magnitude of the 32 rows (so far) is at most 448 * 2^E: the values of a head's 32 rows keep their four significant bits down to 2^-13 of the largest
 * one's magnitude.
 */
typedef struct {
    void *k, *v;                 /* device, codes [pages, Hkv, block_rows, D], 16-byte aligned */
    unsigned char *k_scales, *v_scales;   /* device, E + 127, [pages, Hkv, ceil(block_rows / 32)] */
    const int *block_table;      /* NULL: a dense cache, pages = B, entry b's rows in page b; else device int32 [B, max_blocks], as for
                                    tiled_sdpa_fwd_paged: block_rows is then 64, 128, 256, ... */
    int pages, Hkv, block_rows;
    int D;                       /* 64, 96, 128 or 160 */
    int max_blocks;
} tsdpa_cache8;

/*
 * Keys and values of a step's tokens into the cache.
 *
 *   k, v      : tsdpa_rows of [B, S, Hkv, D], of type dtype (TSDPA_F16 or TSDPA_BF16).
 *   kv_lens   : device int32 [B]: rows of each entry before the step.
 *   new_lens  : device int32 [B]: rows after it (tiled_sdpa_cache_step): token i of entry b is row new_lens[b] - S + i, and is written if that is
 *               kv_lens[b] or more (entries with fewer than S new tokens have them at the end), and below the capacity (block_rows, or
 *               max_blocks * block_rows).  new_lens[b] <= kv_lens[b], as of a refused step or a drop: nothing is written for the entry.
 *
 * Why lengths and not slots: the tokens that share a scale have to be known together.  Of each block of 32 rows that gets a token, E becomes the
 * least that its new rows need, or, if rows of the block lie below kv_lens[b], what it was if that is more.  Where it grows, these rows
 * keep their values: their codes become code * 2^(old E - new E), rounded (exact but for codes that leave the normal range, below 2^-6).
 * (E of a block falls only when its rows are written from the first on, new: dropped rows leave it as it is.)  Values go to the nearest
 * code, of two equally near ones to that with the even mantissa; magnitudes beyond 448 * 2^62 to the largest, NaN and infinities to NaN,
 * and neither counts for E.  Rows from new_lens[b] on are left as they are, byte for byte; so is what other entries hold, as long as no
 * page is in two entries.  A page number that is none (below 0 or from `pages` on) is not written to.  (B * Hkv * (S / 32 + 2) is below 2^25.)  The cache must not overlap the inputs.
 *
 * Validation order, of all calls of this section: null structs, dtype, D, shape, empty problem, null pointers, alignment, strides, scale,
 * splits, workspace, launch.
 */
int tiled_sdpa_cache8_write(const tsdpa_cache8 *c, const tsdpa_rows *k, const tsdpa_rows *v, const int *kv_lens, const int *new_lens,
                            int B, int S, int dtype, void *stream);

/*
 * Rows of the cache, back in 16 bits: what the calls over a 16-bit cache take, or tokens that are to be written to other rows (the accepted
 * path of a tree: read it, then write it behind the rows from before the tree).
 *
 *   slots        : device int32 [B, n] (as of tiled_sdpa_cache_step): page * block_rows + row in the page.  A slot that is negative or past
 *                  the last page's gives zeros.
 *   k_out, v_out : [B, Hkv, n, D], of type dtype, 16-byte aligned; must overlap neither each other nor the cache.  code * 2^E is exact in
 *                  both types but for what lies outside of FP16's range (below 2^-14, from 65520 on: rounded).
 *   c            : block_table and max_blocks are not looked at; block_rows may be any number; pages * block_rows fits an int.
 */
int tiled_sdpa_cache8_read(const tsdpa_cache8 *c, const int *slots, void *k_out, void *v_out, int B, int n, int dtype, void *stream);

/*
 * Attention over the cache: tiled_sdpa_fwd_kvcache (c->block_table NULL) or tiled_sdpa_fwd_paged on the values that the codes stand for.
 *
 *   q, o         : [B, H, Sq, D], of type dtype, contiguous, 16-byte aligned; H % Hkv == 0, query head h reads head h / (H / Hkv).
 *   lse          : NULL or FP32 [B, H, Sq].
 *   kv_lens      : device int32 [B], rows of each entry, clamped to [0, capacity]; of a dense cache NULL = all of them hold block_rows.
 *   flags        : TSDPA_FLAG_CAUSAL (the queries are the last Sq positions: needs a capacity of Sq or more) or 0.
 *   splits, workspace : as for tiled_sdpa_fwd_kv; 0 = at most tiled_sdpa_cache8_default_splits of the capacity, and no more than the workspace
 *                  has room for.  tiled_sdpa_kv_workspace_bytes(B, H, Sq, D, n) bytes hold n.  B * H * ceil(Sq / 16), times splits, is at
 *                  most 2^23 - 16.
 *   o, lse and the workspace must overlap neither each other nor what the call reads.
 *
 * Scores and sums are FP32.  K is multiplied as 16-bit numbers of q's type, which its codes are; the weights, each times its scale of V, are rounded to
 * FP16 for the product with V: to 11 bits down to 2^-21 of the greatest such product of the row, to multiples of 2^-31 of it (at most) below.  That is by scale, not by
 * value: where a row weighs blocks alike, those with a scale of 2^22 or more below the greatest lose bits, from 2^32 on all, even in columns in which the greatest's block
 * has zeros.  (The normaliser, and so LSE, has all weights in FP32.)
 * A row that no key reaches gets O = 0 and LSE = -infinity, one with a score that is NaN O = LSE = NaN, whatever the number of splits.  Keys that a row does not see do not reach it, NaN among their values included.
 * Page numbers that are none count as the nearest one that is.
 */
int tiled_sdpa_fwd_cache8(const tsdpa_cache8 *c, const void *q, void *o, float *lse, const int *kv_lens, int B, int H, int Sq, float scale,
                          int dtype, unsigned flags, int splits, void *workspace, unsigned long long workspace_bytes, void *stream);

int tiled_sdpa_cache8_default_splits(int B, int H, int Hkv, int Sq, int Skv, int D, int dtype, unsigned flags, int *splits);

/*
 * Measurement aid, not part of the attention path: enqueue a register-resident stream of
 * v_mfma_f32_32x32x16 (FP16 or BF16 per `dtype`) on every SIMD of the GPU -- 512 workgroups of four
 * wavefronts, `iters` x 64 MFMAs per wavefront -- so the caller can time what the matrix pipe
 * sustains with no memory traffic.  random_operands != 0 fills the operand registers with random
 * signs and mantissas (the switching activity of real data, under which the chip lowers its
 * clock); 0 uses constant ones; 2 is the random-operand stream with the rest of the attention
 * loop's instruction mix added at the loop's own ratios and independent of the MFMAs (per MFMA one
 * 16-byte-per-lane LDS read and 3.7 vector instructions, a quarter of them exponentials): the rate
 * that mix sustains when nothing ever waits for anything.  sink: device buffer of at least 512*256 floats, overwritten.
 * flops (host pointer, may be NULL) receives the flop count of the launch.  The Section 4.2.3
 * policy of measuring on an otherwise idle GPU applies.  Returns a status code; iters = 0 only
 * reports flops (nothing is launched and sink may then be NULL; with iters > 0 a NULL sink is
 * TSDPA_ERR_NULL_PTR).
 */
int tiled_sdpa_probe_mfma(int dtype, int random_operands, int iters, float *sink, double *flops,
                          void *stream);

/*
 * Measurement aid, not part of the attention path: enqueue a kernel that reads `bytes` of device memory at
 * `src` once (8192 workgroups, each a contiguous run, four 16-byte loads per lane in flight) and writes
 * nothing but one word per workgroup into `sink` (device, at least 512*256 floats).  What a decoding step
 * (Section 7: reading the K/V cache once is all it does) can be compared with besides the published
 * HBM figure: the rate a pure read stream sustains on this GPU.  src: device, 16-byte aligned; bytes: at
 * least 128 MiB (smaller is refused as a bad shape), the part that does not fill a whole loop trip of every
 * workgroup is not read; bytes_read (host pointer, may be NULL) receives the bytes the launch does read.
 * Returns a status code.
 */
int tiled_sdpa_probe_hbm_read(const void *src, unsigned long long bytes, float *sink, double *bytes_read,
                              void *stream);

/* Human-readable text for a status code (static storage, never NULL). */
const char *tiled_sdpa_status_string(int status);

/* Library version: major * 10000 + minor * 100 + patch. */
int tiled_sdpa_version(void);

#ifdef __cplusplus
}
#endif
#endif /* TILED_SDPA_H */
