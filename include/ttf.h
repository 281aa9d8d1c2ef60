/*
 * ttf.h -- C ABI of the Temporal Token Fusion (TTF) pre-LLM compression pass for AMD
 * Instinct MI355X (gfx950).
 *
 * TTF (paper Section 3, "Temporal Token Fusion") takes the visual tokens of a clip,
 * X in R^{FN x C} viewed as [F, N=H*W, C], and
 *   1. picks an anchor frame a: the frame whose mean token has the largest cosine with the
 *      clip's mean token (anchor-frame-selection equation), or a caller-fixed frame
 *      (ablation A2: first / last frame);
 *   2. for every token (k,i) of every other ("source") frame searches the (2r+1)x(2r+1)
 *      neighbourhood of its grid cell in the anchor frame, clamped to the grid with
 *      duplicate cells counted once, for the anchor token of largest cosine similarity:
 *      best similarity s^(k,i) and anchor flat index dst(k,i) (pointwise matching with
 *      local window search: projection, flat-index map, similarity, arg max, s^/dst);
 *   3. fuses the token (drops it; the anchor token at dst stands for it) iff s^ > t, keeps
 *      it iff s^ <= t (threshold-gating equation);
 *   4. emits the compressed sequence X' = [N anchor rows ; P kept source rows in ascending
 *      flat order k*N+i] as bit-exact copies of input rows (no averaging), together with
 *      each row's original position triple (k, y, x) (stacked-X' equation, positional
 *      alignment: mask, gather of X and P) and the compressed length L' = N + P that
 *      cache-aware decode alignment needs.
 *
 * A batch holds B independent clips: every clip gets its own anchor, matches, mask and
 * L'; outputs are packed clip after clip.  (The paper's tied-batch rule -- one offset from
 * the batch-mean similarity, keep = union over the batch -- is a different mode, offered by
 * ttf_compress_tied.)
 *
 * General conventions
 *   - All data pointers are DEVICE pointers unless a field says HOST.  Every buffer is
 *     owned by the caller, before, during and after the call.  The library allocates and
 *     frees no device memory.
 *   - Work is enqueued on the caller's stream and the call returns without synchronising.
 *     Buffers must stay alive until the stream has drained.  Calls that share a workspace
 *     must be ordered by the caller (same stream, or events).
 *   - Every function returns a ttf_status.  On any status other than TTF_OK no kernel has
 *     been launched and no output has been written, except TTF_ERR_HIP, which reports a
 *     failed launch or copy part-way through the sequence (outputs are then undefined).
 *   - Same inputs give bit-identical outputs on every call (no floating-point atomics, fixed
 *     reduction orders).
 *   - Input values are not scanned.  A candidate whose cosine is NaN (a NaN or infinite entry in
 *     the source token or in that anchor token) wins no comparison.  A source token all of whose
 *     candidates are like that is kept and reports best_sim = -inf, best_idx = -1, fuse_map = -1.
 *     A NaN or infinite entry anywhere in a clip makes every anchor score NaN; the automatic
 *     rule then picks frame 0.  Dot products and squared norms are accumulated in fp32: token rows
 *     whose squared norm overflows fp32 (entries around 1e17 and beyond) behave like rows with
 *     infinite entries.  Only an exactly zero norm gives cosine 0.
 */
#ifndef TTF_H
#define TTF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    TTF_OK = 0,
    TTF_ERR_INVALID_ARG = 1,          /* NULL required pointer, size <= 0, r < 0, non-finite t, ... */
    TTF_ERR_UNSUPPORTED = 2,          /* unknown dtype, misaligned features / tokens_out            */
    TTF_ERR_WORKSPACE_TOO_SMALL = 3,  /* workspace_bytes < ttf_workspace_size()                     */
    TTF_ERR_HIP = 4                   /* a HIP call failed; see ttf_last_hip_error()                */
} ttf_status;

typedef enum { TTF_BF16 = 0, TTF_F32 = 1 } ttf_dtype;

typedef enum { TTF_ANCHOR_AUTO = 0, TTF_ANCHOR_FIXED = 1 } ttf_anchor_mode;

/* Problem description.  B*F*ceil(H*W/64)*64 (the token count with every frame rounded up to whole
 * 64-token groups) must be below 2^25 = 33 554 432, and H*W below 2^31. */
typedef struct {
    int32_t B, F, H, W, C;    /* clips, frames, token-grid height and width, channels; all >= 1 */
    int32_t dtype;            /* ttf_dtype of `features` and `tokens_out`                        */
    int32_t r;                /* search radius >= 0, window (2r+1)^2; r >= max(H,W)-1 = whole grid */
    float   t;                /* cosine threshold; fused iff s^ > t (strict).  Any finite value.  */
    int32_t anchor_mode;      /* ttf_anchor_mode                                                  */
    int32_t anchor_index;     /* FIXED only: frame in [-F, F); negative counts from the last     */
} ttf_params;

/*
 * Outputs.  cap = B*F*H*W rows is the capacity the row-indexed buffers must have; rows at
 * and beyond row_offsets[B] are left untouched.  N = H*W.
 */
typedef struct {
    void*    tokens_out;    /* [cap, C] dtype.  Clip b owns rows row_offsets[b] .. row_offsets[b+1)-1:
                               first its N anchor rows, then its kept source rows (stacked-X' equation). */
    int32_t* pos_ids;       /* [3, cap] planes k (frame), y, x of every output row (plane stride cap). */
    int32_t* src_index;     /* [cap]    flat index k*N+i inside its clip of every output row (I_keep). */
    int32_t* row_offsets;   /* [B+1]    exclusive prefix sum of kept_count.                            */
    int32_t* kept_count;    /* [B]      L'_b = N + P_b.                                                */
    int32_t* anchor_index;  /* [B]      anchor frame chosen (or given) per clip.                       */
    int32_t* fuse_map;      /* [B,F,N]  dst(k,i) in [0,N) if the token was fused, else -1
                                        (anchor-frame tokens: -1).                                     */
    float*   best_sim;      /* [B,F,N]  s^(k,i); 1.0f on anchor-frame tokens.  May be NULL.            */
    int32_t* best_idx;      /* [B,F,N]  dst(k,i) for every source token whether fused or not;
                                        i on anchor-frame tokens.  May be NULL.                        */
    int32_t* host_counts;   /* HOST, pinned, [2B+1]: kept_count[0..B) then row_offsets[0..B]; filled by
                               an asynchronous copy on the stream.  May be NULL.                       */
} ttf_outputs;

/* Bytes of device workspace ttf_compress needs for these sizes (depends on B,F,H,W,C and dtype only).
 * The workspace must be 256-byte aligned.  INVALID_ARG on bad sizes or NULL pointers. */
ttf_status ttf_workspace_size(const ttf_params* params, size_t* bytes);

/*
 * The whole pass (Section 3: anchor frame selection, pointwise matching with local window
 * search, threshold gating and token compression, positional alignment).
 *   features   DEVICE [B,F,H,W,C] contiguous, dtype per params, 16-byte aligned; read only.
 *   workspace  DEVICE scratch of at least ttf_workspace_size() bytes, 256-byte aligned; its
 *              contents on entry do not matter and are garbage afterwards.
 *   out        see ttf_outputs; all but the three optional fields are required.
 *   hip_stream hipStream_t (NULL = the default stream).
 * Errors: INVALID_ARG (NULL params/features/workspace/out or required output, a size < 1,
 * more than 2^25 tokens (frames rounded up to 64), r < 0, t not finite, anchor_index outside [-F,F) in FIXED mode, unknown
 * anchor_mode), UNSUPPORTED (unknown dtype; features, tokens_out or workspace misaligned),
 * WORKSPACE_TOO_SMALL, HIP.  Any C, grid and radius work.  Fast paths: bf16 and fp32 input with
 * C % 32 == 0 and r <= 2 runs the window search on the matrix cores (fp32 as three bf16 pieces per
 * value, 24 significant bits) on any grid; grids exactly 16 or 32 tokens wide with H*W % 64 == 0 are
 * the best case.  So do larger bf16 problems with C % 8 == 0 and C >= 768 (see ttf_search_route), for
 * which ttf_workspace_size() asks for more than the other kernels need: a workspace that is only
 * large enough for those, about B*H*ceil(W/16)*16*(C rounded up to 32, minus C)*2 bytes less, is taken too and
 * runs them.  Rows whose byte length is a multiple of 16 are read and copied with 16-byte accesses.
 */
ttf_status ttf_compress(const ttf_params* params, const void* features,
                        void* workspace, size_t workspace_bytes,
                        const ttf_outputs* out, void* hip_stream);

/*
 * ttf_compress for callers that cannot allocate device memory or hand over a workspace: code
 * running under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, outputs and errors as ttf_compress on a workspace of this size, but it is a fixed array of
 * TTF_STATIC_WORKSPACE_BYTES that lives in the library's device image (every GPU the library is
 * used on holds its own copy from the first use until the process ends).  The call allocates and
 * frees nothing.
 *   - Problems whose ttf_workspace_size() exceeds TTF_STATIC_WORKSPACE_BYTES are refused with
 *     TTF_ERR_WORKSPACE_TOO_SMALL before anything is launched.  (bf16 rows with C % 32 != 0 count as they
 *     are; where the room for the matrix-core search of such rows does not fit as well, they take the
 *     general kernels, whose similarities differ in the last bits: see ttf_search_route.)
 *   - All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (two
 *     streams, two threads) race and give undefined outputs; order them on one stream or with events.
 *     The array keeps the previous call's contents; nothing in it needs to start at zero.
 *   - The first call on a device looks up the array's device address (hipGetSymbolAddress); make
 *     that call outside any stream capture.  TTF_ERR_HIP if the lookup fails.
 */
#define TTF_STATIC_WORKSPACE_BYTES (16u << 20)
ttf_status ttf_compress_static(const ttf_params* params, const void* features,
                               const ttf_outputs* out, void* hip_stream);

/*
 * One segment of a stream (the streaming use sketched in Discussion D3): video arrives in pieces, and
 * each piece is matched not against a frame of its own but against the frame that closed the
 * previous piece, so that earlier context never has to be encoded again.
 * Every one of the F frames of `features` is a source frame matched against `anchor_frame`; the
 * output holds only the preserved source rows, in ascending flat order k*N+i, so it is what
 * ttf_compress gives for the (F+1)-frame clip [anchor_frame ; features] with its anchor fixed to
 * frame 0, without the N anchor rows.  To chain segments pass the previous segment's last frame
 * (features + (F-1)*N*C elements of each clip, gathered to [B,H,W,C]) as the next anchor_frame.
 *   anchor_frame  DEVICE [B,H,W,C] dtype, 16-byte aligned, read only; may alias no output
 *   frame_offset  added to the temporal plane of pos_ids: frame k of the segment reports
 *                 frame_offset + k (its index in the stream); frame_offset + F must fit int32
 *   out           as for ttf_compress, except: kept_count[b] = P_b (no anchor rows),
 *                 anchor_index[b] = -1, best_idx / fuse_map index cells of anchor_frame,
 *                 src_index = k*N+i inside the segment
 * params->anchor_mode and anchor_index are not used.  Errors as for ttf_compress; a NULL or
 * misaligned anchor_frame is INVALID_ARG / UNSUPPORTED.  ttf_restore_map does not apply to
 * segment outputs (their anchor rows live in an earlier segment's output).
 */
ttf_status ttf_compress_segment(const ttf_params* params, const void* features, const void* anchor_frame,
                                int32_t frame_offset, void* workspace, size_t workspace_bytes,
                                const ttf_outputs* out, void* hip_stream);

/*
 * Tied-batch mode (Section 3, the remark on B > 1 after the s^/dst equations, and the gating
 * paragraph): the B elements are treated as views of one sequence.  For every source position the
 * candidate cell is scored by the average of the B elements' cosines and one cell is picked for all of
 * them; each element reports its own cosine at that shared cell; a position is dropped only when
 * every element's cosine exceeds t.  All B elements therefore keep the same index set and the
 * output is rectangular.  Choices the text leaves open: the anchor frame is
 * shared -- under the automatic rule the frame with the largest batch-mean anchor score (lowest
 * k on ties), else the fixed frame; the mean is the arithmetic mean of the B cosines of one
 * candidate cell; first maximum in row-major offset order.  Radius r <= 3 (UNSUPPORTED beyond).
 *
 * cap = F*N rows.
 */
typedef struct {
    void*    tokens_out;    /* [B, cap, C] dtype: element b's rows start at row b*cap; rows
                               0..L'-1 of every element are valid, the rest untouched            */
    int32_t* pos_ids;       /* [3, cap] planes k, y, x of the shared rows                         */
    int32_t* src_index;     /* [cap] flat k*N+i of the shared rows                                */
    int32_t* kept_count;    /* [1] L' = N + P                                                     */
    int32_t* anchor_index;  /* [B] every entry = the shared anchor frame                          */
    int32_t* fuse_map;      /* [F,N] shared: dst(k,i) if every element has s^ > t, else -1        */
    float*   best_sim;      /* optional [B,F,N]: s^ of every element at the shared offset (1 on
                               anchor rows)                                                      */
    int32_t* best_idx;      /* optional [F,N]: shared dst(k,i) (i on anchor rows)                 */
    float*   mean_sim;      /* optional [F,N]: the maximal batch-mean similarity (1 on anchor
                               rows)                                                             */
    int32_t* host_counts;   /* optional HOST pinned [1]: copy of kept_count                       */
} ttf_tied_outputs;

/* Workspace bytes of ttf_compress_tied (depends on B,F,H,W,C,dtype and r). */
ttf_status ttf_tied_workspace_size(const ttf_params* params, size_t* bytes);

/* Arguments and errors as for ttf_compress; workspace of ttf_tied_workspace_size() bytes. */
ttf_status ttf_compress_tied(const ttf_params* params, const void* features, void* workspace,
                             size_t workspace_bytes, const ttf_tied_outputs* out, void* hip_stream);

/*
 * Restoration (Discussion D4, token restoration through the map dst(k,i) of the matching step).
 *
 * ttf_restore_map: for every original token, the row of the compressed sequence that stands for
 * it -- its own row if it was retained (anchor tokens included), the anchor row
 * row_offsets[b] + dst(k,i) if it was fused.
 *   fuse_map, row_offsets, src_index   DEVICE, as written by ttf_compress for the same params
 *   restore_map                        DEVICE int32 [B,F,N], every entry written
 * ttf_restore: the full layout rebuilt from the compressed rows,
 *   restored[b,k,i,:] = tokens[restore_map[b,k,i], :]   (bit-exact row copies).
 *   tokens       DEVICE [rows, C] dtype, 16-byte aligned (ttf_compress's tokens_out, or rows of the
 *                same shape computed from it, e.g. after further layers)
 *   rows         number of valid rows in `tokens`; map entries outside [0, rows) give a zero row
 *   restored     DEVICE [B,F,N,C] dtype, 16-byte aligned
 * Errors: INVALID_ARG (NULL pointer, bad sizes, rows < 0), UNSUPPORTED (dtype, alignment), HIP.
 */
ttf_status ttf_restore_map(const ttf_params* params, const int32_t* fuse_map, const int32_t* row_offsets,
                           const int32_t* src_index, int32_t* restore_map, void* hip_stream);
ttf_status ttf_restore(const ttf_params* params, const void* tokens, int64_t rows,
                       const int32_t* restore_map, void* restored, void* hip_stream);

/*
 * Cache-aware decode alignment (Section 3; prefill-length and decode-position equations), host
 * arithmetic on HOST integers: with L' compressed visual tokens and T text tokens the cache holds
 * L_pre = L' + T pairs; decode step l = 0,1,... gets position L_pre + l and an attention mask of
 * length L_pre + l + 1.  Output pointers may be NULL.  INVALID_ARG on a negative input.
 */
ttf_status ttf_decode_alignment(int64_t l_prime, int64_t text_tokens, int64_t step,
                                int64_t* l_pre, int64_t* position, int64_t* mask_length);

/*
 * Video-adaptive threshold (Discussion D1: t calibrated from the empirical distribution of the
 * best-match similarities of the current clip).  The paper leaves the rule open; this library
 * uses an order statistic.  For a requested fused fraction phi in [0,1] of the M = (F-1)*N source
 * tokens of a clip:  rank = clamp(ceil((1 - phi) * M), 1, M)  (formed in double precision), and
 * thresholds[b] = the rank-th smallest s^ of clip b.  Tokens strictly above it fuse, so at most
 * floor(phi*M) do, exactly that many when the values next to the rank are distinct.  F = 1 gives
 * thresholds[b] = 1.  Values are ordered as real numbers (-0 just below +0; a NaN with the sign
 * bit clear sorts above +inf, with it set below -inf).  Outputs of ttf_compress_segment
 * (anchor_index[b] = -1) work too: all F frames are then source frames, M = F*N.
 *   best_sim, anchor_index   DEVICE, as written by ttf_compress (best_sim requested there)
 *   thresholds               DEVICE float [B]
 * Errors: INVALID_ARG (NULL pointer, bad sizes, phi outside [0,1] or NaN), HIP.
 */
ttf_status ttf_select_threshold(const ttf_params* params, const float* best_sim,
                                const int32_t* anchor_index, float fused_fraction,
                                float* thresholds, void* hip_stream);

/*
 * Gate, offsets and row emission redone from stored matches (threshold-gating equation and the
 * compaction that follows it), without a window search: the result is what ttf_compress gives
 * for the same features with clip b gated at thresholds[b] (or at params->t for every clip when
 * thresholds is NULL) and its anchor fixed to anchor_index[b].
 *   out->anchor_index, out->best_sim, out->best_idx   INPUTS here: DEVICE arrays a previous
 *       ttf_compress on the same features and params (r included) wrote; all three required
 *   out->fuse_map, tokens_out, pos_ids, src_index, row_offsets, kept_count, host_counts   written
 *   thresholds   DEVICE float [B] or NULL
 * params->anchor_mode / anchor_index / r are not used.  Workspace as for ttf_compress.
 */
ttf_status ttf_regate(const ttf_params* params, const void* features, const float* thresholds,
                      void* workspace, size_t workspace_bytes, const ttf_outputs* out, void* hip_stream);

/*
 * From the compressed rows into attention.
 *
 * What a language model does next with the rows, positions and lengths of the pass: norm and rotate queries
 * and keys by the rows' (t, y, x) positions, put keys and values into a paged cache, attend over it.  Rows are
 * packed sequence after sequence, as ttf_compress packs clips: row_offsets may be its output, and pos its pos_ids
 * planes.  dtype, here and there, is a ttf_dtype; sums, norms, angles and softmax statistics are held in 32 bits or more and
 * every output is rounded once.
 *
 * The lengths, offsets, positions and page numbers are device data and are not checked by the host.  Whatever
 * they hold, nothing outside the buffers described is read or written:
 *   - row_offsets has to be non-decreasing and start at 0 or later; entries beyond `rows` count as `rows`.  (With
 *     others the outputs are undefined.)  Rows outside [row_offsets[0], row_offsets[batch]) are left as they were.
 *   - cached[b] < 0: sequence b appends nothing, and its rows attend to nothing.
 *   - The attention sees the entries below 2^31 - 2^20 of a sequence.
 *   - Page-table entries outside [0, pages) are pages that are not there (not yet given out, or given back behind a
 *     window), and so is everything beyond table_width: nothing is appended to them, and their keys are left out of the softmax.
 */
typedef enum { TTF_ROPE_HALF = 0, TTF_ROPE_INTERLEAVED = 1 } ttf_rope_layout;

/*
 * Queries, keys and values of `rows` rows, with the norm and the rotation they get.  Strides are in elements; the
 * entries of a head are contiguous.  Pointers and strides of q, k, v and the outputs are multiples of 16 bytes; no two heads of an
 * output share an entry.
 *
 *   norm     y_i = x_i w_i / sqrt(mean_i x_i^2 + eps) over the head_dim entries of a head, where the weight is given
 *   angle    theta_j = pos[axis[j]][row] * inv_freq[j] for the pairs j < rotary_dim / 2, formed in 64 bits
 *   rotate   (y_a, y_b) -> (y_a c - y_b s, y_b c + y_a s), c = attention_factor cos theta_j, s = attention_factor sin theta_j, taken in 64
 *            bits and rounded to 32 once,
 *            (a, b) = (j, j + rotary_dim/2) with TTF_ROPE_HALF, (2j, 2j+1) with TTF_ROPE_INTERLEAVED; entries from
 *            rotary_dim on are not rotated
 */
typedef struct {
    int32_t dtype;                  /* of q, k, v, the weights and the outputs                                    */
    int32_t head_dim;               /* D: a multiple of 8, at most 256                                            */
    int32_t heads, kv_heads;        /* of q; of k and v                                                           */
    int32_t rows, batch;            /* rows of the buffers; sequences.  Up to 2^24 rows, 2^20 sequences           */
    const int32_t* row_offsets;     /* [batch+1] first row of every sequence.  ttf_qk_norm_rope: NULL = all rows  */
    const int32_t* cached;          /* [batch] pairs already in the cache (ttf_cache_append only)                 */
    const void *q, *k, *v;          /* [rows, heads, D], [rows, kv_heads, D] by the strides                       */
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;
    void *q_out, *k_out;            /* may be q and k themselves (same strides), otherwise must not overlap them  */
    int64_t qo_row, qo_head, ko_row, ko_head;
    const void *q_weight, *k_weight;   /* [D] norm weights; NULL = no norm                                        */
    float eps;                      /* >= 0, finite                                                               */
    int32_t rotary_dim;             /* R: even, 0 <= R <= D; 0 = no rotation (pos and inv_freq may be NULL)       */
    int32_t layout;                 /* ttf_rope_layout                                                            */
    int32_t axes;                   /* position planes, 1 to 4                                                    */
    const double* inv_freq;         /* [R/2]                                                                      */
    const int32_t* axis;            /* [R/2] plane of every pair, NULL = 0; entries outside [0, axes) count as 0  */
    const int32_t* pos;             /* [axes, rows] planes pos_stride entries apart                               */
    int64_t pos_stride;
    float attention_factor;
} ttf_qk_params;

/* A paged cache: page p, slot s, head h of k (and of v) starts at element p*page_stride + s*slot_stride +
 * h*head_stride; entry t of sequence b is slot t % page_size of page page_table[b*table_stride + t / page_size].
 * Pointers and strides of k and v are multiples of 16 bytes; no two heads of a page share an entry where it is written. */
typedef struct {
    void *k, *v;
    const int32_t* page_table;      /* [batch, table_width]                                     */
    int64_t page_stride, slot_stride, head_stride, table_stride;
    int32_t pages, page_size, table_width;
} ttf_kv_cache;

/*
 * Frequencies of a rotation, host arithmetic on HOST arrays: inv_freq[j] = base^(-2j/R) of the R/2 pairs, R = rotary_dim,
 * slowed down for contexts longer than the model was trained on (original_length positions):
 *   TTF_ROPE_PLAIN    as they are
 *   TTF_ROPE_LINEAR   all divided by factor
 *   TTF_ROPE_BASE     base * factor^(R/(R-2)) in the place of base: the first pair stays, the last is divided by factor
 *   TTF_ROPE_PARTS    divided by factor to a share g_j in [0,1]: f (1 - g) + f / factor g, with g growing linearly in j from 0 to 1
 *                     between the pairs that turn `fast` and `slow` times over original_length positions (the first rounded
 *                     down, the second up, neither below 0; beyond the last pair where all turn faster than that: the last is then
 *                     divided in part, or not at all); attention_factor = 0.1 ln(factor) + 1
 *   TTF_ROPE_TURNS    the same with 1 - g linear in the number of turns between slow and fast; attention_factor = 1
 * and axis[j], the plane of each pair, from the number of pairs of every plane: sections[axes] (HOST; their sum is R/2; NULL: all
 * plane 0).  take_turns 0: one block of pairs after the other.  Otherwise the planes take turns: pair j goes to plane
 * a = j % axes where a > 0 and j / axes < sections[a], else to plane 0 (there have to be that many pairs).
 * Output pointers may be NULL.  INVALID_ARG: rotary_dim odd or < 2, base <= 1, factor < 1, original_length < 1 where it
 * is used, slow not below fast, a negative section, sections that do not sum to R/2, axes outside 1..4.
 */
typedef enum { TTF_ROPE_PLAIN = 0, TTF_ROPE_LINEAR = 1, TTF_ROPE_BASE = 2, TTF_ROPE_PARTS = 3, TTF_ROPE_TURNS = 4 } ttf_rope_scaling;
ttf_status ttf_rope_table(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_length, double fast,
                          double slow, int32_t axes, const int32_t* sections, int32_t take_turns, double* inv_freq,
                          int32_t* axis, float* attention_factor);

/*
 * Norm and rotation of queries and keys in one pass: q_out = rotate(norm(q)), k_out = rotate(norm(k)).  q (with heads 0)
 * or k (with kv_heads 0) may be left out; v is not used.
 * Errors: INVALID_ARG (NULL pointer, bad sizes, bad strides, eps), UNSUPPORTED (dtype, head_dim, alignment), HIP.
 */
ttf_status ttf_qk_norm_rope(const ttf_qk_params* params, void* hip_stream);

/*
 * The same, with the keys and the values put into the cache: row i of sequence b (row row_offsets[b] + i of the
 * buffers) becomes entry cached[b] + i.  k_out is not used.  q (heads 0) may be left out; rotated queries go to q_out.
 * Two rows that the page table sends to one slot leave either's entries there, element by element.
 * Errors: as above.
 */
ttf_status ttf_cache_append(const ttf_qk_params* params, const ttf_kv_cache* cache, void* hip_stream);

/*
 * Attention of new rows over the cache they were appended to.  Row i of sequence b has index t = cached[b] + i; of the
 * entries u < cached[b] + row_offsets[b+1] - row_offsets[b] it sees those with u <= t (causal), u > t - window (window > 0),
 * on pages that are there:
 *   out = sum_u w_u v_u,  w = softmax_u(scale <q, k_u>),   lse = ln sum_u exp(scale <q, k_u>)
 * (lse joins parts of a context attended to separately).  A row that sees nothing gets out = 0, lse = -inf.  Query head h reads
 * key head h / (heads / kv_heads).  Entries that a row does not see have no influence on it, whatever bits
 * they hold.  Scores, statistics and sums are in 32 bits.  With bf16, the weights of the sum over v_u are rounded on the way into the matrix
 * cores: to 2^-16 of each, or, where max_rows heads / kv_heads is above 32 (16 with heads of more than 128 entries), to bf16 (2^-8 of each); lse
 * is not touched by that.  Ordinary decoding is the chunk of one row: ttf_decode_alignment's position is cached[b], its mask
 * length the number of entries seen.
 *   max_rows    most rows of a sequence, or any other number from 1 on (below the mean it counts as the mean): it picks the kernel, and
 *               so the order of sums, the rounding of weights and the room in the workspace; no result depends on its being right
 *   workspace   DEVICE, ttf_attention_workspace_size() bytes, 256-byte aligned; contents on entry do not matter.  Calls that may
 *               overlap need one each.  The size is enough for every call with the same dtype, head_dim, heads and kv_heads and
 *               no more rows, batch and max_rows: small calls may take more room than large ones, so a call by itself may need less
 * Errors: INVALID_ARG (NULL pointer, bad sizes, heads no multiple of kv_heads, scale not finite, window < 0), UNSUPPORTED (dtype,
 * head_dim, alignment), WORKSPACE_TOO_SMALL, HIP.
 */
typedef struct {
    int32_t dtype, head_dim, heads, kv_heads;       /* as in ttf_qk_params                             */
    int32_t rows, batch, max_rows;
    int32_t causal, window;                         /* 0 or 1; entries a row looks back over, 0 = all  */
    float scale;
    const int32_t* row_offsets;                     /* [batch+1]                                       */
    const int32_t* cached;                          /* [batch] entries in the cache before these rows  */
    const void* q;                                  /* [rows, heads, D] by the strides                 */
    void* out;                                      /* [rows, heads, D] by the strides; may be q itself, same strides */
    float* lse;                                     /* optional [rows, heads]                          */
    int64_t q_row, q_head, o_row, o_head;
} ttf_attention_params;
ttf_status ttf_attention_workspace_size(const ttf_attention_params* params, size_t* bytes);
ttf_status ttf_paged_attention(const ttf_attention_params* params, const ttf_kv_cache* cache, void* workspace,
                               size_t workspace_bytes, void* hip_stream);

/* Static, NUL-terminated description of a status code (never NULL). */
const char* ttf_status_string(ttf_status status);

/* hipError_t (as int) behind the calling thread's last TTF_ERR_HIP; 0 if none. */
int ttf_last_hip_error(void);

/*
 * How ttf_compress evaluates the automatic anchor rule (the anchor-frame-selection equation needs the
 * mean of every frame, i.e. a pass over the whole input before the search can start).
 *   two-pass      frame sums over the whole input, then the search.
 *   speculative   the rule is first evaluated on 256 of the C channels (four runs of 64 channels,
 *                 run j starting at channel (2j+1)*C/8 rounded down to a multiple of 64).  A clip
 *                 whose guessed best frame beats the runner-up by at least 0.1 in that cosine is
 *                 searched against the guess at once, the search adds up the exact sums of every
 *                 frame on the side, and the exact rule is evaluated from them afterwards: it
 *                 confirms the guess, or the clip is searched again against the exact anchor.
 *                 A clip without a clear guess sits out the first search and takes the two-pass
 *                 route together with the refuted clips.  Outputs are those of the
 *                 exact rule in every case, bit for bit the same as on the two-pass route; only the time
 *                 differs (one pass over the input instead of two when the guesses hold, one extra search
 *                 for a clip whose trusted guess was wrong).
 *                 Available where the search walks whole frames (see ttf_search_route) with C >= 1024, F >= 2
 *                 and the automatic anchor: for fp32 input with C % 32 == 0 and r <= 1, and for bf16 input with
 *                 C % 128 == 0 and r <= 2 on grids whose rows fill at least 70 % of the 32-cell
 *                 strips (two rows each up to 16 columns, one up to 32: 12..16, 23..32, 45..64, ... columns; any
 *                 height); fp32 clips only while the guess, 1 to 8 KiB a frame, fits beside the window products
 *                 (a few frames fewer than walk; many fewer on grids of some dozen tokens).
 * mode  0 (default): speculative where it is expected to be faster (from 256 MiB on, clips of 12 to 128
 *       frames, those of more than 64 only where it is expected to save much; fp32 on grids of up to 16 columns;
 *       depends on B, F, the grid, r and C), and there only if
 *       enough of the clips have a clear guess: else all take the two-pass route;
 *       1: speculative wherever available;  -1: always two-pass.
 * Process-wide; takes effect for calls made after it returns.  INVALID_ARG for other values.
 */
ttf_status ttf_set_speculation(int mode);

/*
 * Which window-search kernels a problem takes (Section 3, "Pointwise Matching with Local Window
 * Search"): a host-side query, no GPU work.  The routes add the channels in different orders:
 * similarities agree to about 3e-7 (each within 1e-5 of the exact value), and only a token whose
 * similarity lies that close to t, or to another candidate's, may be gated or matched differently.
 * So do the kernels behind one route: problems with C >= 1024 (fp32: 768, r <= 1) and whole 128-byte groups of
 * channels take a search that walks whole frames where it is the faster one, which depends on the grid, r, C and the
 * size of the input (bf16 grids exactly 16 or 32 wide with whole keep words: from 24 to 160 MiB on), and where the
 * window products of all its frames have room in the workspace.  They are n * ((2r+1)^2 + 1) floats a token, n = C / 2048
 * (fp32: C / 1024) rounded up; where the speculative route exists for bf16 (see ttf_set_speculation) there is room for any
 * F, elsewhere it is that of the anchor's copy, 2C (fp32: 6C) bytes for every cell of a frame with rows padded to
 * whole 16 columns: 31 frames of 16x20 C 1024 r 2, 54 of 16x16 C 1088 r 1, 153 of fp32 16x16 C 4096 r 1.  A clip one
 * frame too long takes the search it would take below the size lines.  The walk makes fp32 problems of 32 MiB and
 * more matrix-core ones that would otherwise be too small.
 * For most problems the route depends on dtype, r, C and the grid.  For bf16 with C % 32 != 0 (C % 8 == 0,
 * C >= 768) it also depends on B and F -- small problems and few-column grids are searched faster by the
 * general kernels -- and on the workspace: the answer is for one of ttf_workspace_size() bytes (a
 * smaller one that ttf_compress still takes runs the general kernels).  A segment takes the route of the
 * clip it equals: ask with F + 1 frames.
 *   params  host; checked as in ttf_compress.
 *   route   host, out: one of the TTF_ROUTE_* values.
 * Errors: INVALID_ARG (NULL pointer, bad params), UNSUPPORTED (unknown dtype).
 */
#define TTF_ROUTE_GENERAL      0   /* wave-per-token kernels (any C, any radius) */
#define TTF_ROUTE_MFMA_BF16    1   /* matrix cores, bf16, grid exactly 16 or 32 wide with whole keep words */
#define TTF_ROUTE_MFMA_BF16_PADDED 2   /* matrix cores, bf16, any other grid (tile rows padded to 16 columns) */
#define TTF_ROUTE_MFMA_F32     3   /* matrix cores, fp32 as three bf16 pieces per value, any grid */
ttf_status ttf_search_route(const ttf_params* params, int* route);

/*
 * Per-stage timing, for benchmarks.  Stages, in launch order:
 *   0 frame sums (speculative route: over the guess channels only)   1 anchor scores (two-pass
 *     route only)   2 anchor choice + norms   3 window search + gate
 *   4 anchor verification (speculative route only: exact rule from the search's sums, repeated
 *     search of refuted clips)   5 offsets scan (nothing up to 256 keep words, nor up to 4096 with rows of
 *     1 KiB and more: there stage 6 counts the rows itself)   6 row emission
 * ttf_profile_enable(slots), 1 <= slots <= TTF_PROFILE_MAX_SLOTS, makes every following
 * ttf_compress on the calling thread record HIP events around each stage on the call's
 * stream; successive calls use `slots` event sets round-robin (created once, reused), so up to
 * `slots` calls can be in flight or waiting to be read.  ttf_profile_enable(0) turns it off.
 * Enabling resets the call counter.  ttf_profile_read(call, ms_out, n) waits for profiled call
 * number `call` (0-based since enabling; must be one of the last `slots` calls) and writes its
 * stage durations in milliseconds to ms_out[0..min(n, TTF_NUM_STAGES)); stages that did not
 * run report ~0.  Event records sit between the kernels; profiling is off by default.
 * This is a measurement hook, not part of the pass: it is the one place where the library creates
 * HIP objects (events, at most TTF_PROFILE_MAX_SLOTS sets per thread, created by the first
 * ttf_profile_enable that needs them and kept until the process ends); ttf_compress and
 * ttf_compress_segment record into them only while profiling is enabled on the calling thread,
 * the other entry points never do.  Do not enable it around a stream capture.
 * Errors: INVALID_ARG (bad slot count, NULL, call not available), HIP.
 */
#define TTF_NUM_STAGES 7
#define TTF_PROFILE_MAX_SLOTS 256
ttf_status ttf_profile_enable(int slots);
ttf_status ttf_profile_read(int call, float* ms_out, int n);
const char* ttf_stage_name(int stage);

#ifdef __cplusplus
}
#endif
#endif /* TTF_H */
