/*
 * pevlm.h -- C ABI of the B200 (sm_100a) PEVLM prefill-attention library.
 *
 * The method (paper sections in brackets): a long video token stream is laid out as
 *   [ sink | c_0 | c_1 | ... | c_{N-1} | question ]          lengths S, B, .., B, Q
 * with L = S + N*B + Q [Sec. 3.2.1, Sec. 3.2.3].  Every token keeps its original global
 * position for RoPE [Sec. 3.2.2].  With f = softmax(Q K^T / sqrt(d)) V [Eq. 1]:
 *   sink rows      attend causally to the sink                         [Eq. 3]
 *   rows of c_i    attend to the whole sink and causally to c_i        [Eq. 4, Eq. 8]
 *   question rows  attend causally to every token                      [Eq. 5]
 * The sink's K/V are computed once and shared by all blocks [Sec. 1, Sec. 3.1].
 *
 * Conventions the paper leaves open and this library fixes: the diagonal is visible;
 * RoPE rotates the pairs (i, i + d/2); q head h uses kv head h / (Hq/Hkv); LSE is the
 * natural log of the sum of exp(scaled score).
 *
 * General rules for every entry point
 *   - All tensor pointers are DEVICE pointers, contiguous, bf16 (2-byte brain float) unless
 *     stated, and 16-byte aligned; the attention OUTPUT `o` of pevlm_parallel_prefill_attn,
 *     pevlm_block_attn and pevlm_query_attn(_noalloc) must be 32-byte aligned (its rows are
 *     written with 32-byte vector stores; likewise those of the calls below that say so), workspaces 256-byte aligned.  A pointer that misses
 *     its alignment is refused with PEVLM_EALIGN before any launch.  `stream` is a
 *     cudaStream_t passed as void* (NULL = the legacy default stream).  `shape` is a HOST
 *     pointer.  Input values must be finite.
 *   - The caller owns every buffer and the stream.  The library allocates no device
 *     memory, never synchronises the device (pevlm_read_status excepted) and never frees
 *     anything.  Calls are asynchronous on `stream`.  No state is kept between calls, with
 *     one exception: pevlm_query_attn_noalloc owns a fixed device array per GPU and
 *     remembers its address in each context (see there).
 *   - batch > 1 means `batch` independent sequences of the same shape, stored one after
 *     another (the leading dimension of every tensor, and of the workspace partials).
 *   - Return value: PEVLM_OK (0) or a negative pevlm_status_t.  All argument checking
 *     happens before any launch; nothing aborts, traps or throws.  Device-side waits are
 *     bounded: if one expires the kernel records PEVLM_ETIMEOUT in the first word of the
 *     workspace and finishes; read it with pevlm_read_status after the stream is idle.
 */
#ifndef PEVLM_H_
#define PEVLM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PEVLM_OK = 0,
    PEVLM_EINVAL = -1,       /* bad shape or NULL pointer */
    PEVLM_EALIGN = -2,       /* a pointer misses its alignment (16 bytes; attention outputs 32; workspaces 256) */
    PEVLM_EUNSUPPORTED = -3, /* head_dim not in {64,128}, device is not sm_100, ... */
    PEVLM_EWORKSPACE = -4,   /* workspace NULL or too small */
    PEVLM_ECUDA = -5,        /* a CUDA call failed; text via pevlm_last_cuda_error */
    PEVLM_ETIMEOUT = -6      /* a bounded device-side wait expired (see pevlm_read_status) */
} pevlm_status_t;

typedef enum {
    PEVLM_MASK_PEVLM = 0,      /* Eq. 3-5: sink + own block */
    PEVLM_MASK_FULL_CAUSAL = 1 /* plain causal attention over the video tokens (Eq. 1-2) */
} pevlm_mask_mode_t;

typedef struct {
    int32_t batch;         /* >= 1 */
    int32_t sink_len;      /* S >= 0 tokens  [Sec. 3.2.1 "Sink Block"] */
    int32_t block_len;     /* B >= 1 if num_blocks > 0  [uniform "Context Blocks"] */
    int32_t num_blocks;    /* N >= 0 */
    int32_t query_len;     /* Q >= 0  ["Question Block"] */
    int32_t num_q_heads;   /* Hq */
    int32_t num_kv_heads;  /* Hkv, Hq % Hkv == 0 */
    int32_t head_dim;      /* d in {64, 128} */
    float rope_theta;      /* RoPE base, e.g. 1e4 or 1e6 */
    float softmax_scale;   /* 0 => 1/sqrt(d)  [Eq. 1] */
    int32_t mask_mode;     /* pevlm_mask_mode_t */
} pevlm_shape_t;

typedef enum {
    PEVLM_WS_PREFILL = 0, /* workspace of pevlm_parallel_prefill_attn */
    PEVLM_WS_QUERY = 1    /* workspace of pevlm_query_attn and of the question in pevlm_layer_forward */
} pevlm_workspace_kind_t;

/*
 * RoPE at global positions [Sec. 3.2.2].  Rotates every head vector of q_in
 * [n_tokens, Hq, d] and k_in [n_tokens, Hkv, d] by the angles pos * theta^(-2i/d),
 * i < d/2, pairing elements (i, i+d/2), where pos = pos_ids[t] if pos_ids != NULL (device
 * int32[n_tokens]) else first_token + t.  Angle, sine/cosine and rotation are evaluated in
 * fp64; the result is rounded once, fp64 -> fp32 -> bf16, round-to-nearest-even.  Results
 * go to q_out / k_out (same shapes); out may equal in (in place) or be any other buffer
 * (for K: the slot of these tokens in the KV cache).  Either (q_in,q_out) or (k_in,k_out)
 * may both be NULL to skip that tensor.  batch applies to all four tensors and to pos_ids.
 */
int pevlm_rope_qk(const pevlm_shape_t* shape, const void* q_in, const void* k_in, void* q_out,
                  void* k_out, int64_t first_token, int64_t n_tokens, const int32_t* pos_ids,
                  void* stream);

/*
 * pevlm_rope_qk and, in the same launch, the copy of the same tokens' V rows: v_in [n_tokens, Hkv, d] to v_out (for
 * instance the slot of these tokens in the V cache); a NULL pair skips that tensor as it does for Q and K, of which one
 * must be given.  batch applies to all six tensors.
 */
int pevlm_rope_qkv(const pevlm_shape_t* shape, const void* q_in, const void* k_in, const void* v_in, void* q_out,
                   void* k_out, void* v_out, int64_t first_token, int64_t n_tokens, const int32_t* pos_ids,
                   void* stream);

/*
 * Multimodal RoPE: the model family the paper evaluates encodes temporal and spatial coordinates in its
 * position embedding (Sec. 3.1), so every token has three position
 * components, pos_ids3 = device int32 [3, n_tokens] (temporal, height, width).  Rotary pair i < d/2 takes
 * its position from component 0 for i < sections[0], from component 1 for the next sections[1] pairs and
 * from component 2 for the last sections[2] (host int32[3], sum = d/2; the split itself is the model's,
 * not the paper's, e.g. {16, 24, 24} at d = 128).  Sequential positions in the sense of Sec. 3.2.2 means
 * the ids are those of the unpartitioned stream.  Everything else as pevlm_rope_qk (fp64 evaluation, one
 * rounding, in place or out of place, NULL pairs skipped); batch applies to pos_ids3 as [batch, 3, n_tokens].
 */
int pevlm_rope_qk_mrope(const pevlm_shape_t* shape, const void* q_in, const void* k_in, void* q_out,
                        void* k_out, int64_t n_tokens, const int32_t* pos_ids3, const int32_t* sections,
                        void* stream);

/*
 * Prefill attention of the video tokens [Eq. 3, Eq. 4]: rows [0, S + N*B).
 *   q [S+N*B, Hq, d], k, v [S+N*B, Hkv, d]  (q, k already roped), read only
 *   o [S+N*B, Hq, d] bf16, lse [Hq, S+N*B] fp32 (may be NULL), written
 * With mask_mode = PEVLM_MASK_FULL_CAUSAL the same kernel computes plain causal
 * attention over the S+N*B tokens.  Only the tiles a query tile can see are visited.
 * workspace: >= pevlm_workspace_bytes(shape, PEVLM_WS_PREFILL) bytes, 256-byte aligned.
 */
int pevlm_parallel_prefill_attn(const pevlm_shape_t* shape, const void* q, const void* k,
                                const void* v, void* o, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream);

/*
 * Attention of a range of context blocks against a resident cache [Eq. 4 for those blocks alone]: the
 * num_blocks blocks of block_len tokens whose roped K and V sit at rows [first_key_row, first_key_row + N*B)
 * of k_cache / v_cache [cache_rows, Hkv, d]; rows [0, S) of the cache are the sink.  Each block sees the
 * sink and itself causally, exactly as in pevlm_parallel_prefill_attn; the sink rows are not recomputed.
 *   q_blocks [N*B, Hq, d] roped, o [N*B, Hq, d], lse [Hq, N*B] (may be NULL): the block rows only.
 * Because blocks do not attend to one another (Sec. 1), this one call serves (i) a video whose length is
 * not a multiple of the block length (Sec. 3.2.1 partitions uniformly and is silent on a remainder: the
 * remainder is taken as one shorter last block, run with block_len = its length), (ii) a streaming window
 * that encodes one new block against the fixed sink into any free slot of the cache (the paper's
 * future work, Sec. 5), (iii) per-sequence shapes, one call per shape.  mask_mode must be
 * PEVLM_MASK_PEVLM; first_key_row >= S and first_key_row + N*B <= cache_rows, else PEVLM_EINVAL.
 * batch strides: N*B rows for q / o / lse, cache_rows rows for the caches.  Workspace as for
 * pevlm_parallel_prefill_attn.  Only cache rows [0, S) and the block range are read: a ragged last key tile
 * takes zeros, not the neighbouring rows, past the end of either range, so the rest of the cache may hold
 * anything (uninitialised slots of a streaming window included).
 */
int pevlm_block_attn(const pevlm_shape_t* shape, const void* q_blocks, const void* k_cache,
                     const void* v_cache, int64_t first_key_row, int64_t cache_rows, void* o, float* lse,
                     void* workspace, size_t workspace_bytes, void* stream);

/*
 * KV-cache assembly [Eq. 5's key set s + c_all + q]: k_cache, v_cache [L, Hkv, d] receive
 * the video rows [0, S+N*B) from k_video / v_video and the question rows from k_question /
 * v_question [Q, Hkv, d].  K inputs are roped.  A source pointer may be NULL to skip that
 * part (for instance when pevlm_rope_qk already wrote K into the cache).
 */
int pevlm_assemble_kv(const pevlm_shape_t* shape, const void* k_video, const void* v_video,
                      const void* k_question, const void* v_question, void* k_cache,
                      void* v_cache, void* stream);

/*
 * Question attention [Eq. 5]: the Q question rows attend to cache rows [0, S+N*B) and
 * causally to the question rows themselves (cache rows S+N*B ..).  Split over the key
 * range; partials are merged by their log-sum-exp.
 *   q_question [Q, Hq, d] roped; k_cache, v_cache [L, Hkv, d]
 *   o [Q, Hq, d] bf16, lse [Hq, Q] fp32 (may be NULL)
 * workspace: >= pevlm_workspace_bytes(shape, PEVLM_WS_QUERY) bytes, 256-byte aligned; those of a shape are enough for shorter
 * questions and caches too.
 */
int pevlm_query_attn(const pevlm_shape_t* shape, const void* q_question, const void* k_cache,
                     const void* v_cache, void* o, float* lse, void* workspace,
                     size_t workspace_bytes, void* stream);

/*
 * Question attention without a caller workspace.  (The paper has no counterpart to this entry
 * point; it exists for deployment.)
 *
 * For callers that cannot allocate device memory where they need this step -- code inside a
 * memory-planned or real-time region that must not call cudaMalloc or any allocating library
 * routine, or a plug-in that is handed inputs and outputs but owns no memory pool.  Same
 * arguments, results and errors as pevlm_query_attn, minus the workspace: the split-KV partials
 * go to a fixed array of PEVLM_NOALLOC_SCRATCH_BYTES that is part of the library image, so
 * every GPU that loads the library holds that much device memory until the process exits.
 *   - Shapes whose partials exceed that size are rejected
 *     with PEVLM_EWORKSPACE before any launch (text via pevlm_last_cuda_error).
 *   - The call itself performs no cudaMalloc / cudaFree and uses no allocating routine.
 *   - The first call in each context (one per device, as a rule) resolves the array's device address
 *     (cudaGetSymbolAddress, with that device current); make that first call outside any
 *     stream capture.
 *   - All calls on one device share the one array, which keeps the previous call's contents:
 *     each call clears the status header it needs on the stream and overwrites the partials it
 *     reads.  Two calls whose kernels overlap on the GPU (different streams, no ordering
 *     between them) race on the array; order them.
 *   - A device-side timeout is left in the array's header; pevlm_read_status with
 *     workspace = NULL reads it back (for the current device).
 */
#define PEVLM_NOALLOC_SCRATCH_BYTES (32u << 20)
int pevlm_query_attn_noalloc(const pevlm_shape_t* shape, const void* q_question, const void* k_cache,
                             const void* v_cache, void* o, float* lse, void* stream);

/*
 * The whole pass of one layer over one sequence [Sec. 3.2; Eq. 3-5], from un-roped q [L, Hq, d], k, v [L, Hkv, d]: RoPE at
 * global positions with K and V written to the caches, the prefill attention of the video rows (or full causal) and the
 * question attention.  The same results as pevlm_rope_qk, pevlm_assemble_kv, pevlm_parallel_prefill_attn and
 * pevlm_query_attn in that order (the question's key splits differ, so its sums may differ in their last bits), in two or three
 * launches: the work items of both attention steps share one, so that neither leaves SMs idle.
 *   q_video [S+N*B, Hq, d], q_question [Q, Hq, d]: roped copies (scratch); k_cache, v_cache [L, Hkv, d], o_*, lse_*: written.
 *   last_len > 0: the last of the num_blocks blocks has only that many tokens (<= block_len), L and S+N*B accordingly.
 * batch must be 1.  Pointers of an empty part (no video rows, no question) may be NULL.  Workspaces as for the two attention
 * calls; ws_query must have pevlm_workspace_bytes(shape, PEVLM_WS_QUERY) bytes.
 */
int pevlm_layer_forward(const pevlm_shape_t* shape, int32_t last_len, const void* q, const void* k, const void* v,
                        void* q_video, void* q_question, void* k_cache, void* v_cache, void* o_video, float* lse_video,
                        void* o_question, float* lse_question, void* ws_prefill, size_t ws_prefill_bytes,
                        void* ws_query, size_t ws_query_bytes, void* stream);

/*
 * Attention under a sliding window beside the first tokens, which stay visible (the streaming use of Sec. 5 by tokens instead of blocks):
 * rows [first_token, first_token + n_tokens) of a sequence against its keys; row p sees key j <= p if j > p - window (its own position
 * counts) or j < sink_len (of shape).  One call serves a whole prefill (first_token = 0), a chunk of one behind a cache, and single
 * tokens (few rows take a kernel of their own, like those of pevlm_query_attn).
 *   q [n_tokens, Hq, d] roped; k_cache, v_cache [cache_rows, Hkv, d], of which rows [0, first_token + n_tokens) may be read
 *   (cache_rows >= that; rows that no row of the call sees are not read: they may hold anything); o [n_tokens, Hq, d] (32-byte aligned), lse [Hq, n_tokens] (may be NULL)
 * batch > 1: sequences of equal lengths, n_tokens rows of q and o, cache_rows rows of the caches apart.  Of `shape` batch, sink_len, the head
 * counts, head_dim and softmax_scale are used.  window >= 1; first_token + n_tokens <= 2^30.
 * workspace: >= pevlm_window_workspace_bytes(...) bytes, 256-byte aligned; that of a call does for any first_token and window.
 */
int pevlm_window_attn(const pevlm_shape_t* shape, int32_t window, const void* q, const void* k_cache, const void* v_cache,
                      int64_t first_token, int64_t n_tokens, int64_t cache_rows, void* o, float* lse, void* workspace,
                      size_t workspace_bytes, void* stream);

/* Bytes of workspace of pevlm_window_attn (0 if an argument is invalid). */
size_t pevlm_window_workspace_bytes(const pevlm_shape_t* shape, int32_t window, int64_t first_token, int64_t n_tokens);

/* ---- A cache of many sequences: pages, and keys and values in 4 bits -------------------------------------------------
 *
 * (The paper has no counterpart: it stops at the cache of one video.  These calls are for a server that keeps several
 * videos resident and answers questions about them, Eq. 5 over a cache in pages.)
 *
 * The tokens of a sequence live in pages of page_len tokens, found through its row of the page table: token t at slot
 * page_table[sequence][t / page_len] * page_len + t % page_len.  Pages that no sequence holds stand on a free list, a stack of which the
 * first *free_count entries count.  Lengths, tables, list and count are DEVICE int32, so that a step whose lengths only the GPU
 * knows can be captured into a graph; int32 pointers need 4-byte alignment, `slots` and `positions` 16-byte.
 */
typedef struct {
    int32_t num_pages; /* pages there are, num_pages * page_len < 2^31 */
    int32_t page_len;  /* tokens of a page: 16, 32, 64 or 128 */
    int32_t num_seqs;  /* sequences: rows of the page table */
    int32_t max_pages; /* columns of the page table, max_pages * page_len <= 2^30 */
} pevlm_pages_t;

/*
 * Gives the pages of finished sequences back: for every sequence r with finished[r] != 0, in order, its
 * ceil(lens[r] / page_len) pages are pushed onto the free list, and its length becomes 0.
 *   finished, lens [num_seqs], page_table [num_seqs, max_pages], free_count [1]: read
 *   free_list [num_pages]: written from entry *free_count on; lens_out [num_seqs], free_count_out [1]: written
 * Outputs must not share memory with inputs or with one another (PEVLM_EINVAL): a step goes lens -> release -> lens_out -> assign -> lens.  The page table
 * stays as it is: what stands behind a sequence's length means nothing.  Lengths and counts outside their range count as the
 * nearest one inside; nothing is written past the end of the free list.
 */
int pevlm_pages_release(const pevlm_pages_t* pages, const int32_t* finished, const int32_t* lens, const int32_t* page_table,
                        int32_t* free_list, const int32_t* free_count, int32_t* lens_out, int32_t* free_count_out, void* stream);

/*
 * Room for new_lens[r] >= 0 more tokens of every sequence: pages taken from the top of the free list in the order of the
 * sequences (the j-th page taken by all of them is free_list[*free_count - 1 - j]), and for each new token, the rows of all sequences
 * one after another, its slot and its position.
 *   lens, new_lens [num_seqs], free_list, free_count: read; page_table: entries of fresh pages written
 *   lens_out [num_seqs] = lens + new_lens, free_count_out [1]
 *   row_start [num_seqs + 1]: first row of each sequence, and the number of rows at the end
 *   slots, positions [max_rows]: written in full, rows that no sequence has with slot -1 and position 0.  (positions is the pos_ids
 *   of pevlm_rope_qk, slots those of pevlm_packed_store, lens_out and row_start those of pevlm_packed_attn; where a
 *   sequence may be turned away, key_lens of pevlm_pages_assign_rows in place of lens_out.)
 * A sequence whose pages run out (the free list, counted over all sequences up to this one, or its row of the table) or
 * whose rows end past max_rows gets no pages: its rows have slot -1 and its lens_out stays lens.  One that needs no fresh page is never
 * turned away for the list.  Outputs, the page table among them, must not share memory (see pevlm_pages_release).  max_rows >= 0, <= 2^30.
 */
int pevlm_pages_assign(const pevlm_pages_t* pages, const int32_t* lens, const int32_t* new_lens, int32_t* page_table,
                       const int32_t* free_list, const int32_t* free_count, int32_t* lens_out, int32_t* free_count_out,
                       int32_t* row_start, int32_t* slots, int32_t* positions, int64_t max_rows, void* stream);

/*
 * The same for a step that brings n_rows rows, 0 <= n_rows <= max_rows, whatever new_lens says: a sequence whose rows end past n_rows is
 * turned away like one whose rows end past max_rows.  (Granted, it would hold tokens that nobody has written, i.e. what the pages'
 * former sequences left there.)  slots and positions are written up to max_rows all the same.
 *   key_lens [num_seqs], may be NULL: lens_out, but 0 for a sequence that was turned away.  As the lens of pevlm_packed_attn it leaves the rows
 *   of such a sequence without keys: output 0 and LSE -inf, where lens_out would place them at the end of what the sequence held before.
 */
int pevlm_pages_assign_rows(const pevlm_pages_t* pages, const int32_t* lens, const int32_t* new_lens, int32_t* page_table,
                            const int32_t* free_list, const int32_t* free_count, int32_t* lens_out, int32_t* free_count_out,
                            int32_t* row_start, int32_t* slots, int32_t* positions, int64_t max_rows, int64_t n_rows, int32_t* key_lens,
                            void* stream);

/*
 * The packed cache: K and V in groups of 16 values along the head, each value an e2m1 number (4 bits: 0, 0.5, 1, 1.5, 2, 3, 4, 6
 * and their negatives) times the e4m3 scale of its group; 4.5 bits a value.  For a group with largest magnitude m
 *   scale = e4m3(clamp(m / 6, 2^-9, 448)),  value = e2m1(x / scale), both to nearest, halfway to the even code, the second saturating,
 * so values up to 2688 are in range, and those of a group below 2^-9 * 6 share the smallest scale.  Every value of the cache is a
 * bf16 and an fp16 number: reading it back rounds nothing.  (The sign of a zero is left open: a value that rounds to 0 may be stored as either of the two codes.)
 *   cache [num_pages, Hkv, page_len / 16, 18 * d] bytes: per 16 tokens ("tile") of a page and kv head, token u = 8 h + k, element e:
 *     K codes   byte u * d/2 + e/2                             (element 2i in the low half of its byte)
 *     V codes   byte 8 d + ((h * 8 + c) * 8 + k) * d/16 + b      byte b of eighth c of the head (d/8 elements)
 *     K scales  byte 16 d + k * 2n + (i / w) * 2w + h * w + i % w  group i < n = d/16, w = d/64
 *     V scales  byte 17 d + i * 16 + (k / 2) * 4 + h * 2 + k % 2
 * i.e. in the order in which the threads of the attention's matrix products hold them.
 * pevlm_packed_cache_bytes: bytes of the whole cache (0 if shape or pages are invalid), 16-byte aligned.
 * Of `shape` these calls use num_q_heads, num_kv_heads, head_dim and softmax_scale (and pevlm_packed_attn sink_len); batch must be 1.
 */
size_t pevlm_packed_cache_bytes(const pevlm_shape_t* shape, const pevlm_pages_t* pages);

/*
 * Writes rows into their slots: k, v [n_rows, Hkv, d] bf16, rows k_stride / v_stride elements apart (0 = Hkv * d; a multiple of 8, at
 * least Hkv * d: rows of one projection's output can be taken where they stand), slots [n_rows].
 * A row whose slot is outside [0, num_pages * page_len) is skipped.  Slots must differ: of a slot named twice the contents are a mix.
 */
int pevlm_packed_store(const pevlm_shape_t* shape, const pevlm_pages_t* pages, const void* k, const void* v, int64_t k_stride,
                       int64_t v_stride, const int32_t* slots, int64_t n_rows, void* cache, void* stream);

/* Reads rows back: k_out, v_out [n_rows, Hkv, d] bf16, 32-byte aligned, receive what the cache holds at slots [n_rows] (any order, any of them more than
 * once); zeros for a slot out of range. */
int pevlm_packed_load(const pevlm_shape_t* shape, const pevlm_pages_t* pages, const void* cache, const int32_t* slots, int64_t n_rows,
                      void* k_out, void* v_out, void* stream);

/*
 * Attention of the last rows of every sequence over the packed cache [Eq. 5 for many sequences; single tokens, drafted tokens and
 * question blocks in one call].  Sequence r has lens[r] keys in the cache and rows row_start[r] .. row_start[r + 1] - 1 of q; its i-th
 * of n rows is its token lens[r] - n + i, whose own key is in the cache already, and sees the keys up to its own.  With window > 0
 * only those of the last `window` positions (its own among them) and of the sequence's first sink_len tokens (shape); window = 0: all.  (A window bounds
 * what a row reads, not what a sequence holds: pages in front of it go back with the sequence's others, pevlm_pages_release.)
 *   q [n_rows, Hq, d] bf16 roped, rows q_stride elements apart (0 = Hq * d); lens [num_seqs], row_start [num_seqs + 1], page_table: as
 *   pevlm_pages_assign leaves them;  o [n_rows, Hq, d] bf16, lse [Hq, n_rows] fp32 (may be NULL), written
 *   max_rows: most rows of one sequence, as the caller knows it (n_rows if not): chooses the kernels, which takes time if it is far too large; a larger
 *   row count than that stays correct
 * A row that sees no key (a length of 0, or fewer keys than rows) has output 0 and LSE -inf; so have those of a sequence whose rows end past
 * n_rows, i.e. are not all there.  Keys in a page whose table entry is outside
 * [0, num_pages) count as not there, and what keys hold that no row sees (behind the length, in front of the windows) does not matter.  Rows of q that no sequence has are not read, and of o and lse not written.  Scores of finite rows are formed from fp16
 * operands (the cache's values are exact in it, and of a row of q what is at least 2^-31 of its largest element; what is smaller is off by 2^-39 of that at
 * most) and summed in fp32, probabilities rounded to fp16.
 * workspace: >= pevlm_packed_workspace_bytes(...) bytes, 256-byte aligned, needs no value; two calls at a time need two.
 */
int pevlm_packed_attn(const pevlm_shape_t* shape, const pevlm_pages_t* pages, int32_t window, const void* q, int64_t q_stride,
                      const void* cache, const int32_t* page_table, const int32_t* lens, const int32_t* row_start, int64_t n_rows,
                      int64_t max_rows, void* o, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace of pevlm_packed_attn (0 if an argument is invalid). */
size_t pevlm_packed_workspace_bytes(const pevlm_shape_t* shape, const pevlm_pages_t* pages, int64_t n_rows, int64_t max_rows);

/* Bytes of workspace the given call needs for this shape (0 if the shape is invalid). */
size_t pevlm_workspace_bytes(const pevlm_shape_t* shape, int which /* pevlm_workspace_kind_t */);

/*
 * Reads the status word a kernel may have left in `workspace` (device pointer; NULL = the
 * built-in array of pevlm_query_attn_noalloc on the current device).  Blocks the calling host
 * thread until `stream` is idle.  *status = PEVLM_OK or PEVLM_ETIMEOUT; *detail (may be NULL)
 * = wait id * 1000000 + index of the thread block whose wait expired.
 */
int pevlm_read_status(const void* workspace, void* stream, int32_t* status, int32_t* detail);

/*
 * Self-test of the failure path (the paper has no counterpart): launches one thread block that
 * waits, with the library's bounded wait, on a barrier nothing ever arrives on, until every wait has
 * given up and limit_ns (1 us .. 100 ms) have passed; the kernel records PEVLM_ETIMEOUT with wait id 99 in the
 * header of `workspace` (>= 256 bytes, 256-byte aligned) and ends normally; the context stays
 * usable and the next call on the same workspace clears the status.  Nothing traps or faults.
 */
int pevlm_selftest_wait_expiry(void* workspace, size_t workspace_bytes, int64_t limit_ns, void* stream);

/*
 * Executed tensor-core work of a call for this shape, for throughput accounting:
 * *tiles = number of (query tile, key tile) MMAs pairs visited over all heads and batch,
 * *flops = 4 * d * sum over visited tiles of (tile rows * tile key columns issued).
 */
int pevlm_tile_stats(const pevlm_shape_t* shape, int which, int64_t* tiles, double* flops);

const char* pevlm_strerror(int code);
/* Text of the last CUDA error seen by this thread inside the library ("" if none). */
const char* pevlm_last_cuda_error(void);

#ifdef __cplusplus
}
#endif
#endif /* PEVLM_H_ */
