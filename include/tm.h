/*
 * tm.h -- C ABI of the sparse causal streaming attention library for MI355X
 * (gfx950): the attention of the chunked autoregressive video-diffusion student
 * of TalkingMachines (arXiv 2506.03099) and the KV-cache append that lets its
 * denoising steps reuse cached context.
 *
 * The operation (paper Sec. 4.2, "Chunked Processing", "Sparse Attention
 * Pattern" and the attention equation; Sec. 4.3, "KV & Embedding Cachings"):
 * the latent sequence is a run of latent frames of T tokens each; the first R
 * frames form the starting chunk c_0 (the reference image), the following
 * frames are grouped C at a time into chunks c_1, c_2, ... (the last group may
 * be shorter). A query token of chunk c_a attends, bidirectionally, to every
 * token of c_0 and of c_{a-W} .. c_a (the paper: W = 1, i.e. c_0, c_{t-1},
 * c_t), with exact softmax(q k^T * scale) v over that key set.
 *
 * Conventions shared by every entry point
 *  - Tensors are dense, row-major, in the descriptor's dtype (fp32 or
 *    bfloat16): activations are [B, L, H, D] (batch, token, head, head_dim),
 *    i.e. token stride H*D, head stride D. Every device pointer must be
 *    16-byte aligned and point into device memory that covers the whole
 *    tensor; the library checks both before launching anything.
 *  - The caller owns all device memory and all streams. The library never
 *    allocates or frees device memory and never synchronises a stream: every
 *    launch is asynchronous on the stream passed in, so the caller orders an
 *    append before the attention that reads it (same stream, or events).
 *  - Errors: every status is TM_OK (0) or negative. All argument checks run
 *    on the host before any launch, so an error leaves caches and outputs
 *    untouched. tm_last_error() returns a thread-local message for the last
 *    failing call on that thread. No C++ exception crosses this ABI.
 *  - Threading: thread-compatible; one cache handle must not be used by two
 *    threads at once.
 */
#ifndef TM_H
#define TM_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h> /* hipStream_t */

#ifdef __cplusplus
extern "C" {
#endif

typedef enum tm_status {
    TM_OK = 0,
    TM_E_ARG = -1,      /* null/misaligned pointer, pointer not covering its tensor, bad value */
    TM_E_SHAPE = -2,    /* unsupported or inconsistent sizes */
    TM_E_DTYPE = -3,    /* unknown dtype */
    TM_E_ORDER = -4,    /* chunk index out of streaming order */
    TM_E_CAPACITY = -5, /* more tokens than the chunk (or cache) holds */
    TM_E_DEVICE = -6    /* HIP runtime reported an error */
} tm_status;

typedef enum tm_dtype { TM_F32 = 0, TM_BF16 = 1 } tm_dtype;

#define TM_MAX_WINDOW 12 /* largest supported W */

/* Problem statement of one attention layer (paper Sec. 4.2). All sizes are
 * token or frame counts, never bytes. */
typedef struct tm_attn_desc {
    int32_t batch;            /* B >= 1: independent streams processed together */
    int32_t heads;            /* H >= 1 */
    int32_t head_dim;         /* D: 64 or 128 */
    int32_t tokens_per_frame; /* T >= 1: latent tokens per latent frame */
    int32_t chunk_frames;     /* C >= 1: latent frames per chunk after c_0 */
    int32_t ref_frames;       /* R >= 1: latent frames in c_0 (reference image) */
    int32_t window;           /* W in [0, TM_MAX_WINDOW]: previous chunks seen (paper: 1) */
    int32_t dtype;            /* tm_dtype of q, k, v, o; accumulation is always fp32 */
    float softmax_scale;      /* > 0, or <= 0 for 1/sqrt(D) (the paper's 1/sqrt(d)) */
} tm_attn_desc;

/* Opaque KV cache handle: host-side bookkeeping only (descriptor, the two
 * caller-owned pools, latest chunk index, valid length of each slot). */
typedef struct tm_kv_cache tm_kv_cache;

/* Capacity of one cache in token rows per (batch, head), or 0 if the
 * descriptor is invalid. c_0 is given RC = R*T rounded up to a multiple of 8
 * rows, each of the W+1 ring slots CC = C*T rounded up to a multiple of 8, and
 * the total RC + (W+1)*CC is rounded up to a multiple of 64 (the V pool's
 * block). */
int64_t tm_kv_cache_tokens(const tm_attn_desc* desc);

/* Bytes of ONE pool (the K pool or the V pool) of one cache:
 * B * H * tm_kv_cache_tokens(desc) * D * sizeof(dtype), or 0 if invalid.
 * c_0 occupies token rows [0, R*T) and ring slot s rows [RC + s*CC, ...).
 * K pool layout: [B, H, capacity, D], i.e. each head's cached keys are one
 * contiguous run of D-element rows.
 * V pool layout: [B, H, capacity/64, D, 64]: token rows in blocks of 64, each
 * block stored dimension-major (element (row t, dim d) of a head at
 * (t/64)*64*D + d*64 + t%64), so that 8 consecutive keys of one dimension are
 * 16 contiguous bytes (the attention kernel's V^T operand). */
size_t tm_kv_cache_bytes(const tm_attn_desc* desc);

/* Create a cache over caller-allocated device pools of tm_kv_cache_bytes()
 * bytes each (16-byte aligned). The pools' contents are not read until
 * appended to. On success *out receives the handle (free it with
 * tm_kv_cache_destroy); on error *out is left unchanged. */
tm_status tm_kv_cache_create(const tm_attn_desc* desc, void* k_pool, void* v_pool,
                             tm_kv_cache** out);

/* Release the host-side handle (the pools stay the caller's). NULL is a no-op. */
void tm_kv_cache_destroy(tm_kv_cache* cache);

/* Forget every appended chunk, so the next append must be chunk 0 (a new
 * stream). Launches nothing. */
tm_status tm_kv_cache_reset(tm_kv_cache* cache);

/* Where chunk `chunk` currently lives: its first token row in the pools and
 * its valid length. TM_E_ORDER if the chunk was never appended or has been
 * evicted. Launches nothing. */
tm_status tm_kv_cache_locate(const tm_kv_cache* cache, int32_t chunk, int32_t* token_offset,
                             int32_t* n_tok);

/* Index of the latest appended chunk, or -1 for an empty cache. */
int32_t tm_kv_cache_latest(const tm_kv_cache* cache);

/* KV append / evict (paper Sec. 4.3, "KV & Embedding Cachings": the K/V of
 * c_0 and of c_{t-1} are kept so that context is never recomputed).
 * Copies the new chunk's keys and values, k and v: device [B, n_tok, H, D],
 * into the cache: chunk 0 into the c_0 rows, chunk t >= 1 into ring slot
 * (t-1) mod (W+1). Writing a slot evicts, in place, the chunk t-W-1 it held.
 * Order: the first append after create/reset must be chunk 0; afterwards
 * `chunk` must equal the latest chunk (its K/V are replaced, e.g. by the next
 * denoising step's when one cache is shared by the steps) or latest + 1
 * (advance). Otherwise TM_E_ORDER. n_tok in [1, R*T] for chunk 0 and
 * [1, C*T] for later chunks, else TM_E_CAPACITY. The bit patterns are copied
 * exactly; in the V pool the rows from n_tok up to the next multiple of 8 of
 * the chunk's region are set to zero (they are read, and masked, by the
 * attention kernel's 8-key groups). Bookkeeping is updated only when the
 * launch succeeded. */
tm_status tm_kv_append(tm_kv_cache* cache, int32_t chunk, const void* k, const void* v,
                       int32_t n_tok, hipStream_t stream);

/* Fused K/V producer: RMS normalisation of the chunk's queries and keys, and
 * the KV append, in one launch. The student keeps the attention of its
 * WAN2.1 teacher (paper Sec. 4.1), which normalises queries and keys by their
 * root mean square before the attention equation of Sec. 4.2; the keys cached
 * for later chunks (Sec. 4.3) are those normalised keys. Each (token, head)
 * row x of D elements of q and of k becomes
 *     y[d] = x[d] / sqrt(mean_d(x^2) + eps) * gain[h][d],
 * computed in fp32 and rounded to the cache dtype (nearest even for bf16).
 * q, k, v: device [B, n_tok, H, D] in the cache's dtype, as from the QKV
 * projection. q_out: device, same shape; receives the normalised queries (it
 * may be q itself, but must not otherwise overlap q, k, v or the pools).
 * q_gain, k_gain: device fp32 [H, D] (16-byte aligned), or NULL for ones.
 * eps: finite, >= 0 (TM_E_ARG otherwise). The normalised keys and the values
 * v go into the cache exactly as tm_kv_append would put k and v (same chunk
 * order rules, capacities, layouts, zero padding of V and bookkeeping): the
 * values are copied bit for bit. Replaces a separate normalisation pass and
 * tm_kv_append. */
tm_status tm_qkv_produce(tm_kv_cache* cache, int32_t chunk, const void* q, const void* k,
                         const void* v, const float* q_gain, const float* k_gain, float eps,
                         void* q_out, int32_t n_tok, hipStream_t stream);

/* Sparse causal attention forward (paper Sec. 4.2, attention equation, over
 * the key set {c_0, c_{a-W}, ..., c_a} of the query's chunk a).
 *
 * Streaming form (cache != NULL; k, v must be NULL, n_frames 0): q holds the
 * queries of the latest appended chunk, q_chunk must equal
 * tm_kv_cache_latest(cache) (else TM_E_ORDER), q is [B, n, H, D] with n that
 * chunk's appended length; every key comes from the cache (append the
 * current chunk's K/V first).
 *
 * Full-sequence form (cache == NULL): k, v are [B, n_frames*T, H, D] holding a
 * whole sequence; q_chunk = -1 means q holds all n_frames*T queries
 * (q [B, n_frames*T, H, D]); q_chunk = a >= 0 means q holds only chunk a's
 * queries (q [B, len(a), H, D]).
 *
 * o: device, same shape and dtype as q, written for every query row; it may
 * be q itself (in place) but must not otherwise overlap q, k or v.
 * lse: optional (NULL to skip) fp32 [B, H, Lq], 4-byte aligned: natural-log
 * softmax normaliser log(sum_j exp(scale * q.k_j)) of every query row.
 * Keys outside the allowed set are never read. The result is deterministic
 * (no atomics): repeated calls give identical bits. */
tm_status tm_sparse_causal_attn_fwd(const tm_attn_desc* desc, const void* q, int32_t q_chunk,
                                    const tm_kv_cache* cache, const void* k, const void* v,
                                    int32_t n_frames, void* o, float* lse, hipStream_t stream);

/* The same attention, with the output stored as fp32 instead of the
 * descriptor's dtype (paper Sec. 4.2, the attention equation; for callers
 * that keep the attention output in fp32, e.g. to add it to an fp32 residual
 * stream). Arguments, checks and launch are those of
 * tm_sparse_causal_attn_fwd, except o: device fp32 [B, Lq, H, D], 16-byte
 * aligned. For TM_BF16 inputs the arithmetic is the same kernel's, and only
 * the final rounding of O/l to bf16 (nearest even) is left out, so rounding o
 * to bf16 gives the bf16 call's output bit for bit; o then must not overlap q
 * at all. For TM_F32 inputs this is tm_sparse_causal_attn_fwd (o may be q). */
tm_status tm_sparse_causal_attn_fwd_f32out(const tm_attn_desc* desc, const void* q,
                                           int32_t q_chunk, const tm_kv_cache* cache,
                                           const void* k, const void* v, int32_t n_frames,
                                           float* o, float* lse, hipStream_t stream);

/* The same two calls (o_f32 = 0 or 1: o as in the first or the second) with a
 * caller-owned workspace for the call's duration on `stream`. Query tiles that
 * do not fill the GPU share their keys out in parts, each with a running max of
 * its own, whose results (fp32 O, max and row sum) are merged in a fixed order.
 * Which calls do so, and how, follows from the arguments' sizes alone. With a
 * workspace the parts run on several workgroups and their results go through
 * it; without, they run one after the other. The result is the same, bit for
 * bit.
 * workspace: device memory, 16-byte aligned, not overlapping any other tensor,
 * or NULL. With fewer than tm_sparse_causal_attn_fwd_workspace() bytes (0: the
 * call needs none; also on invalid arguments) it is not used. */
size_t tm_sparse_causal_attn_fwd_workspace(const tm_attn_desc* desc, int32_t q_chunk,
                                           const tm_kv_cache* cache, int32_t n_frames);
tm_status tm_sparse_causal_attn_fwd_ws(const tm_attn_desc* desc, const void* q, int32_t q_chunk,
                                       const tm_kv_cache* cache, const void* k, const void* v,
                                       int32_t n_frames, void* o, int32_t o_f32, float* lse,
                                       void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Backward pass of the full-sequence form (training the student through the
 * attention of Sec. 4.2): given dO = dL/dO, the gradients
 *   dV = P^T dO, dS = P * (dO V^T - rowsum(dO * O)), dQ = scale dS K,
 *   dK = scale dS^T Q,
 * with P the masked row softmax recomputed from lse. Only allowed (query, key)
 * pairs are visited (the same tile skipping as the forward).
 * q, k, v, o, dout: device bf16 [B, L, H, D] with L = n_frames * T, as in the
 * full-sequence forward with q_chunk = -1 (o is its output).
 * lse: device fp32 [B, H, L], the forward's natural-log normaliser (4-byte
 * aligned). delta: caller-owned device fp32 workspace [B, H, L], overwritten
 * with rowsum(dO * O). dq, dk, dv: device bf16 [B, L, H, D], every row
 * written; they must not overlap each other or any input.
 * TM_BF16 only (else TM_E_DTYPE). Three launches on `stream`; deterministic
 * (no atomics). */
tm_status tm_sparse_causal_attn_bwd(const tm_attn_desc* desc, int32_t n_frames, const void* q,
                                    const void* k, const void* v, const void* o, const float* lse,
                                    const void* dout, float* delta, void* dq, void* dk, void* dv,
                                    hipStream_t stream);

/* The same backward pass with a caller-owned workspace for the call's duration
 * on `stream`, taken and checked as in tm_sparse_causal_attn_fwd_ws: tiles that
 * do not fill the GPU (c_0's keys, which every query sees, above all) then share
 * their sums out over several workgroups, whose fp32 parts a fourth launch adds
 * up in a fixed order. That is another order of the fp32 sums than without a
 * workspace: the results of the two calls differ by its rounding (here and there
 * in the last bit of the bf16 gradients), each is deterministic. */
size_t tm_sparse_causal_attn_bwd_workspace(const tm_attn_desc* desc, int32_t n_frames);
tm_status tm_sparse_causal_attn_bwd_ws(const tm_attn_desc* desc, int32_t n_frames, const void* q,
                                       const void* k, const void* v, const void* o, const float* lse,
                                       const void* dout, float* delta, void* dq, void* dk, void* dv,
                                       void* workspace, size_t workspace_bytes, hipStream_t stream);

/* The same backward pass without the caller's workspace, for callers that
 * cannot allocate device memory (code under HIP graph capture, serving loops
 * or harnesses that forbid allocation): delta lives in a device-global array
 * of the library, 8 MiB per GPU (room for B * H * L <= 2^21 rows), which each
 * GPU the library runs on holds until the process ends. Arguments, checks,
 * launches and results, bit for bit, are those of tm_sparse_causal_attn_bwd
 * without delta (not of tm_sparse_causal_attn_bwd_ws where that uses its
 * workspace); B * H * L above 2^21 returns TM_E_CAPACITY. The call allocates
 * nothing. Every call on one GPU uses that GPU's one array (each call writes delta
 * before reading it): calls that overlap in time on one GPU, on different
 * streams or from different threads, race and give wrong gradients; order
 * them. */
tm_status tm_sparse_causal_attn_bwd_noalloc(const tm_attn_desc* desc, int32_t n_frames,
                                            const void* q, const void* k, const void* v,
                                            const void* o, const float* lse, const void* dout,
                                            void* dq, void* dk, void* dv, hipStream_t stream);

/* Number of allowed (query, key) pairs per (batch, head) of the call the same
 * arguments would make (4*D of FLOPs each); -1 on invalid arguments. Pure host
 * arithmetic, launches nothing; the streaming form reads the cache
 * bookkeeping. */
int64_t tm_allowed_pairs(const tm_attn_desc* desc, int32_t q_chunk, const tm_kv_cache* cache,
                         int32_t n_frames);

/* Audio cross-attention with a local frame window and a face mask (paper
 * Sec. 4.1: "Audio Cross Attention with Attention Mask", "Audio Projection
 * Layer", "Speaking/Silence Mode"). Audio tokens are aligned to latent frames,
 * A per frame, covering frames 0 .. F_a - 1; each face has its own audio
 * stream (a silent face's stream holds the special embedding's keys and
 * values). A query token of latent frame f whose face id is m in [0, M)
 * attends, with exact softmax(q k^T * scale) v, to the audio tokens of stream
 * m in frames max(0, f - w) .. min(F_a - 1, f + w) (w = 2: five frames centred
 * on f); a token with any other face id (-1: no face) gets a zero output. */
#define TM_MAX_AUDIO_STREAMS 32

typedef struct tm_audio_desc {
    int32_t batch;            /* B >= 1 */
    int32_t heads;            /* H >= 1 */
    int32_t head_dim;         /* D: 64 or 128 */
    int32_t tokens_per_frame; /* T >= 1: query tokens per latent frame */
    int32_t audio_per_frame;  /* A >= 1: audio tokens per latent frame */
    int32_t audio_frames;     /* F_a >= 1: latent frames the audio covers */
    int32_t streams;          /* M in [1, TM_MAX_AUDIO_STREAMS]: audio streams (faces) */
    int32_t half_window;      /* w >= 0 (paper: 2, a window of five frames) */
    int32_t dtype;            /* TM_BF16 only; accumulation is fp32 */
    float softmax_scale;      /* > 0, or <= 0 for 1/sqrt(D) */
} tm_audio_desc;

/* q: device [B, n_tok, H, D], query row i in latent frame
 * first_frame + i / T; every frame of the run must lie inside the audio
 * (first_frame + ceil(n_tok / T) <= F_a, else TM_E_SHAPE).
 * ak, av: device [B, M, F_a * A, H, D] audio keys and values.
 * face: device int32 [B, n_tok] (4-byte aligned), the stream of each query
 * token; ids outside [0, M) mean no face.
 * o: device [B, n_tok, H, D], every row written; may be q itself (in place)
 * but must not otherwise overlap q, ak, av or face.
 * A frame's window (at most (2w + 1) * A keys, rounded up to 32) must fit in
 * one workgroup's LDS: at most 288 keys at D = 128, 608 at D = 64, else
 * TM_E_SHAPE. n_tok = 0 launches nothing. P is rounded to bf16 before P V;
 * the row sums add the fp32 P. The result is deterministic. */
tm_status tm_audio_cross_attn_fwd(const tm_audio_desc* desc, const void* q, int32_t first_frame,
                                  int32_t n_tok, const void* ak, const void* av,
                                  const int32_t* face, void* o, hipStream_t stream);

/* The same audio cross-attention with the output stored as fp32 (paper
 * Sec. 4.1; for callers that keep the cross-attention output in fp32):
 * arguments and checks as tm_audio_cross_attn_fwd, except o: device fp32
 * [B, n_tok, H, D], 16-byte aligned, not overlapping q. The arithmetic is the
 * bf16 call's; only the final rounding to bf16 (nearest even) is left out,
 * so rounding o to bf16 gives that call's output bit for bit. Rows without a
 * face get zeros. */
tm_status tm_audio_cross_attn_fwd_f32out(const tm_audio_desc* desc, const void* q,
                                         int32_t first_frame, int32_t n_tok, const void* ak,
                                         const void* av, const int32_t* face, float* o,
                                         hipStream_t stream);

/* Rotary positions with three axes (paper Sec. 4.1: the student keeps the
 * attention of its WAN2.1 teacher, whose queries and keys are rotated by the
 * latent frame, row and column of their token before the attention equation of
 * Sec. 4.2). A token at position p of the video lies in latent frame
 * p / (grid_h * grid_w), and in row y and column x of that frame, row-major.
 * The head_dim / 2 pairs of a (token, head) row are shared out over the axes:
 * the first pairs_t turn with the frame, the next pairs_h with the row, the next
 * pairs_w with the column, the rest stay. Pair i of the n pairs of an axis turns
 * by angle = position * theta^(-i / n):
 *     (x0, x1) -> (x0 cos - x1 sin, x0 sin + x1 cos),
 * computed in fp32 and rounded once to the dtype (nearest even for bf16). */
typedef struct tm_rope_desc {
    int32_t head_dim;   /* D: 64 or 128 */
    int32_t frames;     /* >= 1: latent frames the table covers */
    int32_t grid_h;     /* >= 1: tokens per column of a latent frame */
    int32_t grid_w;     /* >= 1: tokens per row; at most 2^30 positions in all, and a table of 2 GiB */
    int32_t pairs_t;    /* >= 0: pairs turned by the frame, */
    int32_t pairs_h;    /* by the row */
    int32_t pairs_w;    /* and by the column; together at most D / 2 */
    int32_t split_half; /* 0: pair i is elements (2i, 2i + 1); else (i, i + D / 2) */
    int32_t dtype;      /* tm_dtype of the rows */
    float theta;        /* > 0 (10000 in the teacher) */
} tm_rope_desc;

/* Bytes of the table of a descriptor, or 0 if it is invalid or turns no pair:
 * (cos, sin) in fp32 of every position and pair, [frames][pairs_t], then
 * [grid_h][pairs_h], then [grid_w][pairs_w]. */
size_t tm_rope3d_table_bytes(const tm_rope_desc* desc);

/* Fill the table: device fp32 of tm_rope3d_table_bytes() bytes, 16-byte aligned;
 * angles, cosines and sines formed in fp64. The caller keeps it as long as calls
 * read it (a table the caller fills itself to that layout does as well). */
tm_status tm_rope3d_table(const tm_rope_desc* desc, float* table, hipStream_t stream);

/* Rotate the queries q: device [batch, n_tok, heads, D] into q_out and the keys
 * k: device [batch, n_tok, kv_heads, D] into k_out, in one launch (k = k_out =
 * NULL and kv_heads = 0: queries only). Row i is the token at position
 * first_token + i, which must lie inside the table's frames (else TM_E_SHAPE).
 * q_out may be q and k_out may be k; no output may overlap anything else.
 * n_tok = 0 launches nothing. */
tm_status tm_rope3d_fwd(const tm_rope_desc* desc, const float* table, int32_t batch, int32_t n_tok,
                        int64_t first_token, const void* q, int32_t heads, const void* k,
                        int32_t kv_heads, void* q_out, void* k_out, hipStream_t stream);

/* Backward pass of tm_rope3d_fwd: given the gradients of its outputs, those of
 * its inputs, dq = R^T dq_out and dk = R^T dk_out (the rotation by the opposite
 * angles). Arguments as in the forward. */
tm_status tm_rope3d_bwd(const tm_rope_desc* desc, const float* table, int32_t batch, int32_t n_tok,
                        int64_t first_token, const void* dq_out, int32_t heads, const void* dk_out,
                        int32_t kv_heads, void* dq, void* dk, hipStream_t stream);

/* The KV cache in 8 bits (paper Sec. 4.3, "KV & Embedding Cachings": the caches
 * of every step and layer stay resident; this one takes half the memory of the
 * 16-bit one and half its traffic). Keys and values are held as 8-bit codes
 * with an fp32 scale for each block of 64 tokens of a chunk and key head, of K
 * and of V apart:
 *     scale = max(m, 2^-60) * fl(1/127),   code = round(x * (1 / scale)),
 * m the largest magnitude in the block, every operation in fp32, rounding to
 * even at ties, so that |code| <= 127 and a value is off by at most about half
 * a scale. It stands for code * scale. A block that holds an infinity or a NaN
 * gets the scale NaN and reads back as NaN throughout.
 * The chunk rules, eviction and key sets are those of tm_kv_cache. Queries, keys
 * and values are bf16 (else TM_E_DTYPE); kv_heads key heads divide the
 * descriptor's heads, query head h reads key head h / (heads / kv_heads). */
typedef struct tm_kv8_cache tm_kv8_cache;

/* Token rows per (batch, key head), or 0 if the descriptor is invalid: c_0 takes
 * R*T rounded up to 64, each of the W+1 ring slots C*T rounded up to 64. */
int64_t tm_kv8_cache_tokens(const tm_attn_desc* desc);

/* Bytes of the pool of one cache, or 0 if invalid: the codes of K, then of V,
 * B * kv_heads * tokens * D bytes each, then the scales of K and of V, one per
 * (batch, key head, block), each rounded up to 16 bytes. Inside a block the codes
 * (as code + 128) are in the order of the attention kernel's operands; use
 * tm_kv8_read for the values. */
size_t tm_kv8_cache_bytes(const tm_attn_desc* desc, int32_t kv_heads);

/* As tm_kv_cache_create, _destroy, _reset, _latest and _locate, over one
 * caller-allocated device pool of tm_kv8_cache_bytes() bytes, 16-byte aligned. */
tm_status tm_kv8_cache_create(const tm_attn_desc* desc, int32_t kv_heads, void* pool,
                              tm_kv8_cache** out);
void tm_kv8_cache_destroy(tm_kv8_cache* cache);
tm_status tm_kv8_cache_reset(tm_kv8_cache* cache);
int32_t tm_kv8_cache_latest(const tm_kv8_cache* cache);
tm_status tm_kv8_cache_locate(const tm_kv8_cache* cache, int32_t chunk, int32_t* token_offset,
                              int32_t* n_tok);

/* Quantise a chunk's k and v, device bf16 [B, n_tok, kv_heads, D], into the
 * cache: order, capacities, eviction and errors as in tm_kv_append. */
tm_status tm_kv8_append(tm_kv8_cache* cache, int32_t chunk, const void* k, const void* v,
                        int32_t n_tok, hipStream_t stream);

/* The producer of tm_qkv_produce for this cache, with the rotary positions of
 * tm_rope3d_fwd in between: queries and keys are RMS-normalised (eps, gains
 * q_gain [heads, D] and k_gain [kv_heads, D] or NULL, as there), rotated (rope
 * NULL: not; table and first_token as in tm_rope3d_fwd, the descriptor's
 * head_dim and dtype those of the cache), and the queries rounded once, to bf16,
 * into q_out: device bf16 [B, n_tok, heads, D] (it may be q; neither it nor the
 * pool may overlap anything else). The keys are quantised from their fp32 values,
 * and the values v as tm_kv8_append does. */
tm_status tm_qkv8_produce(tm_kv8_cache* cache, int32_t chunk, const void* q, const void* k,
                          const void* v, const float* q_gain, const float* k_gain, float eps,
                          const tm_rope_desc* rope, const float* table, int64_t first_token,
                          void* q_out, int32_t n_tok, hipStream_t stream);

/* The keys and values that a cached chunk's codes stand for: code * scale in
 * fp32, into k_out and v_out, device [B, n_tok, kv_heads, D] with n_tok the
 * chunk's appended length, 16-byte aligned; bf16 (nearest even), or fp32 with
 * out_f32 set. TM_E_ORDER if the chunk was never appended or is evicted. */
tm_status tm_kv8_read(const tm_kv8_cache* cache, int32_t chunk, void* k_out, void* v_out,
                      int32_t out_f32, hipStream_t stream);

/* Attention over the 8-bit cache (paper Sec. 4.2, attention equation, over the
 * key set {c_0, c_{a-W}, ..., c_a} of the latest appended chunk a, which q_chunk
 * must name, else TM_E_ORDER): q is device bf16 [B, n_q, heads, D], any number of
 * query rows of that chunk (a whole chunk's, or one token's; 0 launches nothing).
 * o: device, same shape, bf16 or with o_f32 set fp32; written for every row; bf16
 * o may be q itself but must not otherwise overlap anything. lse: optional fp32
 * [B, heads, n_q], 4-byte aligned, natural-log softmax normaliser.
 * Arithmetic: codes and (scaled by a power of two per row) q as fp16 operands,
 * exact but for elements of q below 2^-28 of their row's largest; fp32 sums; P
 * rounded to fp16, of which weights below 2^-18 of the row's largest keep less than
 * 11 bits, to 2^-29 of it; the row sums add the fp32 P. Every dimension has that accuracy
 * whatever the other dimensions' and blocks' sizes, but for values below 2^-60 of the
 * largest that the row sees, which may be off by 2^-60 of that. o_f32 leaves out the
 * final rounding to bf16 only. A query row with an infinity or NaN gets NaN.
 * workspace: device memory, 16-byte aligned, not overlapping any other tensor, or
 * NULL. Rows that do not fill the GPU share their keys out over several
 * workgroups through it; with fewer than tm_kv8_attn_workspace() bytes (0: the call
 * needs none; also on invalid arguments) it is not used, and the fp32 sums are
 * ordered otherwise. Either way the result is deterministic (no atomics). */
size_t tm_kv8_attn_workspace(const tm_kv8_cache* cache, int32_t q_chunk, int32_t n_q);
tm_status tm_kv8_attn_fwd(const tm_kv8_cache* cache, const void* q, int32_t q_chunk, int32_t n_q,
                          void* o, int32_t o_f32, float* lse, void* workspace,
                          size_t workspace_bytes, hipStream_t stream);

/* The rest of a block of the student around its attention (paper Sec. 4.1: the
 * student keeps the blocks of its WAN2.1 teacher, whose branches are normalised,
 * modulated by the timestep's vectors, and gated into the residual stream): the
 * norms before and after a branch, and the linear layers that a branch consists of.
 *
 * Modulations (gates, scales, shifts) are fp32 [B, groups, width], one row for each
 * group of group_tokens tokens (a latent frame; 1: a token): token row i of a call
 * is the token at position first_token + i, of group (first_token + i) /
 * group_tokens, which must be one of the groups (else TM_E_SHAPE); their gradients
 * have zeros for groups without a token in the call. group_tokens = 0: one group,
 * whatever the position. At most 2^20 rows (batch * groups) and 2^30 elements of a modulation. Widths are multiples of 8; fp32 vectors are 16-byte
 * aligned like everything else. No output may overlap anything but where said. Calls that
 * overlap in time (other streams, graphs that run at once) need workspaces of their own. */
typedef enum tm_norm { TM_NORM_NONE = 0, TM_NORM_LAYER = 1, TM_NORM_RMS = 2 } tm_norm;
typedef enum tm_act { TM_ACT_NONE = 0, TM_ACT_GELU = 1, TM_ACT_SILU = 2 } tm_act;

typedef struct tm_block_norm_desc {
    int32_t batch;        /* B >= 1 */
    int32_t width;        /* E: a multiple of 8, at most 16384 */
    int32_t pre;          /* tm_norm of the stream, before the next branch */
    int32_t post;         /* tm_norm of the branch's output y */
    int32_t dtype;        /* tm_dtype of y and h */
    int32_t stream_dtype; /* tm_dtype of x and r */
    int32_t groups;       /* >= 1 */
    int32_t group_tokens; /* >= 1, or 0 with one group */
    float eps;            /* >= 0, of both norms */
} tm_block_norm_desc;

/* Rows of E, all arithmetic in fp32, each output rounded once:
 *     r = x + gate * (post(y) * post_weight)
 *     h = (pre(r) * pre_weight + pre_bias) * (1 + scale) + shift
 * with layer(v) = (v - mean v) / sqrt(var v + eps), rms(v) = v / sqrt(mean v^2 + eps),
 * and r as it is before its rounding. x, r: [B, n_tok, E] in stream_dtype (r may be x
 * itself); y, h: [B, n_tok, E] in dtype; post_weight, pre_weight, pre_bias: fp32 [E];
 * gate, scale, shift: fp32 [B, groups, E].
 * NULL leaves out: y (then r, gate and post_weight are NULL as well, post is
 * TM_NORM_NONE, and x stands for r), gate, any weight, pre_bias, scale and shift (both or neither).
 * With pre TM_NORM_NONE there is no h: it and what belongs to it are NULL. n_tok = 0
 * launches nothing. */
tm_status tm_block_norm_fwd(const tm_block_norm_desc* desc, int32_t n_tok, int64_t first_token,
                            const void* x, const void* y, const float* gate,
                            const float* post_weight, const float* pre_weight,
                            const float* pre_bias, const float* scale, const float* shift, void* r,
                            void* h, hipStream_t stream);

/* Backward pass: from the gradients dh of h and dr of r (what reaches r by other ways; NULL:
 * none, not without pre), those of the inputs: dx (of x; in stream_dtype; may be dr
 * itself), dy (in dtype; may be y or dh itself if y is given), dgate, dscale, dshift (fp32 [B, groups,
 * E]), dpost_weight, dpre_weight, dpre_bias (fp32 [E]). r is the forward's r (x without
 * y), y and the vectors its inputs (shift has no part in it). r and dh are NULL without
 * pre, dy without y. The gradient of a vector that the forward did not have is NULL, and any other
 * one may be (not wanted); dscale and dshift also need scale. Sums over rows are in fp32 and in a fixed order. n_tok = 0 writes zeros to
 * the vectors' gradients.
 * workspace: device memory of tm_block_norm_bwd_workspace() bytes (0 on invalid arguments),
 * 16-byte aligned; needed where a vector's gradient is wanted. */
size_t tm_block_norm_bwd_workspace(const tm_block_norm_desc* desc, int32_t n_tok, int64_t first_token);
tm_status tm_block_norm_bwd(const tm_block_norm_desc* desc, int32_t n_tok, int64_t first_token,
                            const void* r, const void* dh, const void* dr, const void* y,
                            const float* gate, const float* post_weight, const float* pre_weight,
                            const float* pre_bias, const float* scale, void* dx, void* dy,
                            float* dgate, float* dpost_weight, float* dpre_weight, float* dpre_bias,
                            float* dscale, float* dshift, void* workspace, size_t workspace_bytes,
                            hipStream_t stream);

typedef struct tm_linear_desc {
    int32_t batch;        /* B >= 1 */
    int32_t in_width;     /* K: a multiple of 8, at most 2^18 */
    int32_t out_width;    /* N: likewise */
    int32_t act;          /* tm_act; GELU in its tanh form */
    int32_t out_dtype;    /* tm_dtype of o, residual and dout */
    int32_t groups;       /* >= 1, of the gate */
    int32_t group_tokens; /* >= 1, or 0 with one group */
} tm_linear_desc;

/* A linear layer with what follows it:
 *     z = x W^T + bias,   o = residual + gate * act(z)
 * x: bf16 [B, n_tok, K], weight W: bf16 [N, K], bias: fp32 [N], gate: fp32 [B, groups, N],
 * residual, o: [B, n_tok, N] in out_dtype (o may be the residual itself). Sums and
 * everything after them are in fp32, o is rounded once. bias, gate and residual may be
 * NULL; pre, if not NULL, gets z in bf16 [B, n_tok, N], for the backward pass.
 * n_tok = 0 launches nothing. workspace: device memory, 16-byte aligned, or NULL: where
 * tiles leave CUs idle their sums are shared out through it; with fewer than tm_linear_fwd_workspace()
 * bytes (0: the call needs none; also on invalid arguments) they are not, and the fp32
 * sums are ordered otherwise. Either way the result is deterministic. */
size_t tm_linear_fwd_workspace(const tm_linear_desc* desc, int32_t n_tok);
tm_status tm_linear_fwd(const tm_linear_desc* desc, int32_t n_tok, int64_t first_token,
                        const void* x, const void* weight, const float* bias, const float* gate,
                        const void* residual, void* pre, void* o, void* workspace,
                        size_t workspace_bytes, hipStream_t stream);

/* Backward pass: from the gradient dout of o ([B, n_tok, N] in out_dtype, also the
 * residual's gradient), with dz = dout * gate * act'(pre):
 *     dx = dz W (bf16 [B, n_tok, K]),   dweight = dz^T x (bf16 [N, K]),
 *     dbias = sums of dz over rows (fp32 [N]),
 *     dgate = sums of dout * act(pre) over each group's rows (fp32 [B, groups, N]).
 * Any of them may be NULL (not wanted; dgate where the forward had no gate). x is
 * needed for dweight, weight for dx, pre (the forward's, bf16) with an activation and for
 * dgate; else they may be NULL. dz is rounded to bf16 for the two products (with at
 * most 16 rows in all to 16 digits, with at most 4 not at all), sums over rows take it in fp32. All orders are fixed.
 * n_tok = 0 writes zeros to dweight, dbias and dgate. workspace: device memory of
 * tm_linear_bwd_workspace() bytes (0 on invalid arguments, or where none is needed), 16-byte aligned. */
size_t tm_linear_bwd_workspace(const tm_linear_desc* desc, int32_t n_tok, int64_t first_token);
tm_status tm_linear_bwd(const tm_linear_desc* desc, int32_t n_tok, int64_t first_token,
                        const void* x, const void* weight, const void* dout, const float* gate,
                        const void* pre, void* dx, void* dweight, float* dbias, float* dgate,
                        void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Message of the last failing call on this thread ("" if none). */
const char* tm_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* TM_H */
