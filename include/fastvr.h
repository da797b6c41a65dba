/*
 * fastvr.h -- C ABI of the chunk-wise causal attention library (libfastvr.so).
 *
 * The operation is the chunk-wise causal self-attention of FastVR
 * (arXiv 2609.36757, Sec. 3.1, Eq. 1 and the paragraph that follows it):
 * latent tokens, flattened frame-major, are grouped into temporal chunks of
 * `chunk_len` tokens; a query in chunk c sees every key of chunks
 * c - window_chunks .. c (bidirectional inside a chunk, nothing from later
 * chunks).  Eq. 1 is window_chunks = 1; window_chunks = -1 lifts the lower
 * bound (an unbounded causal prefix of chunks).  The same call serves the
 * parallel form over a whole sequence and the streaming form, where one new
 * query chunk attends to a KV cache (q_chunk_offset = that chunk's index
 * relative to the first cached chunk; only chunk differences matter).
 *
 *   LSE_i = ln sum_{j visible to i} exp(scale * q_i . k_j)
 *   O_i   = sum_{j visible to i} exp(scale * q_i . k_j - LSE_i) * v_j
 *
 * Conventions shared by every entry point
 *  - All tensor pointers are DEVICE pointers owned by the caller.  The library
 *    allocates nothing and keeps no pointer after returning.  Its only global
 *    state is a thread-local error string, caches (guarded, safe for concurrent
 *    callers) of each device's CU count and of the last few work plans of the
 *    forward, and the per-device static array of fastvr_chunk_attn_bwd_noalloc.
 *    Every entry point except that one is re-entrant.
 *  - `stream` is a hipStream_t passed as void*; NULL is the null stream.  Calls
 *    return after enqueueing; work is ordered on `stream`.  Faults during
 *    execution surface at the caller's next synchronisation of that stream.
 *  - Every argument is validated on the host BEFORE any HIP call.  A failing
 *    check returns a non-zero status, enqueues nothing, and leaves a message
 *    for fastvr_last_error().  No entry point throws or aborts.
 *  - Element types: bf16 inputs (16-bit brain float, round-to-nearest-even
 *    produced by the caller), fp32 outputs.
 */
#ifndef FASTVR_H
#define FASTVR_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define FASTVR_ABI_VERSION 7

typedef enum {
  FASTVR_OK = 0,
  FASTVR_ERR_INVALID_ARGUMENT = 1, /* null/misaligned pointer, bad size, offset, window, stride or scale */
  FASTVR_ERR_UNSUPPORTED = 2,      /* head_dim not in {64, 128}, or a problem too large for one launch */
  FASTVR_ERR_CAPACITY = 3,         /* a KV append would overflow the cache */
  FASTVR_ERR_HIP = 4               /* the HIP runtime refused a launch */
} fastvr_status;

/*
 * Chunk-causal attention forward (Sec. 3.1, Eq. 1; streaming form: last
 * paragraph of Sec. 3.1).
 *
 *   q   bf16 [B, Nq,  H, d] contiguous     query rows
 *   k   bf16 [B, Nkv, H, d] contiguous     key rows
 *   v   bf16 [B, Nkv, H, d] contiguous     value rows
 *   o   fp32 [B, Nq,  H, d] contiguous     output, fully overwritten
 *   lse fp32 [B, H, Nq]     contiguous     natural-log sum-exp per row, or NULL
 *
 * Query row i lies in chunk q_chunk_offset + i / chunk_len; key row j in chunk
 * j / chunk_len.  Keys of later chunks may be present in k/v; they are masked.
 *
 * Preconditions (else FASTVR_ERR_INVALID_ARGUMENT unless noted):
 *  - q, k, v, o non-NULL and 16-byte aligned; lse NULL or 4-byte aligned;
 *    o does not overlap q, k or v;
 *  - B, H, Nq, Nkv, chunk_len >= 0 and q_chunk_offset >= 0, with
 *    q_chunk_offset * chunk_len + Nq <= Nkv (every query sees its own key, so
 *    no softmax row is empty) and chunk_len >= 1 when Nq > 0;
 *  - d in {64, 128} (else FASTVR_ERR_UNSUPPORTED);
 *  - window_chunks >= -1;  scale finite;
 *  - no element count overflows int64.
 * B, H or Nq equal to 0 is an empty problem: FASTVR_OK, nothing enqueued.
 */
fastvr_status fastvr_chunk_attn_fwd(const void* q, const void* k, const void* v, float* o,
                                    float* lse, int64_t B, int64_t H, int64_t Nq, int64_t Nkv,
                                    int64_t d, int64_t chunk_len, int64_t q_chunk_offset,
                                    int64_t window_chunks, float scale, void* stream);

/*
 * Same operation with explicit element strides, for tensors that are views
 * (e.g. a KV cache [B, capacity, H, d] with capacity > Nkv and B > 1), and a
 * choice of output type: o_bf16 = 0 stores O as fp32, o_bf16 = 1 as bf16 (the
 * fp32 value rounded to nearest even).  Within a token, heads are contiguous
 * with stride d and head_dim elements are contiguous.  Strides are in elements:
 * *_sb between batches, *_st between tokens.  The bf16 strides must be
 * multiples of 8 and the fp32 ones of 4 (16-byte rows), and each must be
 * >= H * d.  lse is [B, H, Nq] contiguous.  o_bf16 not in {0, 1}:
 * FASTVR_ERR_INVALID_ARGUMENT.
 */
fastvr_status fastvr_chunk_attn_fwd_ex(const void* q, int64_t q_sb, int64_t q_st,
                                       const void* k, int64_t k_sb, int64_t k_st,
                                       const void* v, int64_t v_sb, int64_t v_st,
                                       void* o, int64_t o_sb, int64_t o_st, int32_t o_bf16, float* lse,
                                       int64_t B, int64_t H, int64_t Nq, int64_t Nkv, int64_t d,
                                       int64_t chunk_len, int64_t q_chunk_offset,
                                       int64_t window_chunks, float scale, void* stream);

/*
 * KV-cache append for streaming inference with KV caching (Sec. 3.1, last
 * paragraph): copies the new chunk's keys and values
 *   k_new, v_new  bf16 [B, n_new, H, d] contiguous
 * into the caches
 *   k_cache, v_cache  bf16 [B, capacity, H, d] contiguous
 * at token offset cache_len (tokens cache_len .. cache_len + n_new - 1 of each
 * batch).  Nothing is evicted; the caller tracks cache_len.
 * Preconditions: pointers non-NULL and 16-byte aligned, caches not overlapping
 * the new tensors; B, H, capacity, cache_len, n_new >= 0; d in {64, 128};
 * cache_len + n_new <= capacity (else FASTVR_ERR_CAPACITY).
 * n_new, B or H equal to 0: FASTVR_OK, nothing enqueued.
 */
fastvr_status fastvr_kv_cache_append(void* k_cache, void* v_cache, const void* k_new,
                                     const void* v_new, int64_t B, int64_t H, int64_t d,
                                     int64_t capacity, int64_t cache_len, int64_t n_new,
                                     void* stream);

/*
 * Streaming step with a bounded ring KV cache (Sec. 3.1, last paragraph:
 * streaming inference with KV caching, whose cache size stays O(k) for a
 * fixed chunk size k, independent of the video length).  The ring holds
 * W + 1 chunk slots, W = window_chunks (Eq. 1 is W = 1):
 *   k_ring, v_ring  bf16 [B, (W + 1) * chunk_len, H, d] contiguous
 * Chunk c of the stream occupies token rows s * chunk_len .. s * chunk_len +
 * chunk_len - 1 of slot s = c mod (W + 1).  For the new chunk c = chunk_index,
 * given
 *   q_new, k_new, v_new  bf16 [B, n_new, H, d] contiguous   its tokens,
 * one kernel
 *   1. computes the attention of q_new over the keys and values of chunks
 *      max(0, c - W) .. c in chunk order: chunk c from k_new / v_new, the earlier
 *      ones from their ring slots (they must be full chunks written by the
 *      previous steps of the same stream);
 *   2. writes k_new / v_new into slot c mod (W + 1) (the append, fused into the
 *      same launch; the slot held chunk c - W - 1, which chunk c does not see).
 * Outputs o fp32 [B, n_new, H, d] and lse fp32 [B, H, n_new] (or NULL) equal,
 * for the rows of chunk c, those of fastvr_chunk_attn_fwd over the whole
 * sequence with the same window_chunks.
 *
 * Preconditions (else FASTVR_ERR_INVALID_ARGUMENT unless noted):
 *  - all pointers except lse non-NULL and 16-byte aligned, lse NULL or 4-byte
 *    aligned; the ring, o and lse overlap no other argument;
 *  - B, H >= 0; 1 <= n_new <= chunk_len; chunk_index >= 0; 0 <= W;
 *  - W <= 7, d in {64, 128} and chunk_len a multiple of 4 (d = 128) or 8
 *    (d = 64), so that no DMA row group of the kernel straddles two chunks
 *    (else FASTVR_ERR_UNSUPPORTED);
 *  - scale finite; no element count overflows int64.
 * B or H equal to 0: FASTVR_OK, nothing enqueued.
 */
fastvr_status fastvr_chunk_attn_ring_step(const void* q_new, const void* k_new, const void* v_new,
                                          void* k_ring, void* v_ring, float* o, float* lse, int64_t B,
                                          int64_t H, int64_t n_new, int64_t d, int64_t chunk_len,
                                          int64_t chunk_index, int64_t window_chunks, float scale,
                                          void* stream);

/*
 * Backward of fastvr_chunk_attn_fwd (gradients for training with the
 * chunk-causal mask over the whole sequence, Sec. 3.1, Eq. 1), reusing the
 * forward's output and LSE.  With P_ij = exp(scale * q_i . k_j - LSE_i) on
 * visible pairs (0 elsewhere), D_i = sum_c dO_ic O_ic and
 * dS_ij = P_ij (dO_i . v_j - D_i):
 *   dV = P^T dO,   dQ = scale * dS K,   dK = scale * dS^T Q.
 *
 *   q, dout     bf16 [B, Nq,  H, d] contiguous   queries, upstream gradient dL/dO
 *   k, v        bf16 [B, Nkv, H, d] contiguous
 *   o           fp32 [B, Nq,  H, d] contiguous   forward output for (q, k, v)
 *   lse         fp32 [B, H, Nq]     contiguous   forward natural-log LSE
 *   dq          fp32 [B, Nq,  H, d] contiguous   output, fully overwritten
 *   dk, dv      fp32 [B, Nkv, H, d] contiguous   outputs, fully overwritten (zero for
 *                                                keys no query sees)
 *   row_stats   fp32 [B, H, 2, Nq]  contiguous   caller-owned workspace, written by
 *                                                the call: plane 0 LSE_i * log2 e,
 *                                                plane 1 -D_i
 * Mask arguments (chunk_len, q_chunk_offset, window_chunks) and scale are those
 * of the forward call that produced o and lse.  Two kernels run in order on
 * `stream` (row statistics, then all gradients).  Each sum runs in a fixed order,
 * or as two such parts added into a zero, so results are reproducible bit for bit.
 * The two parts are added atomically, which only the device's own coarse-grained
 * memory defines: a call whose dq, dk or dv lie elsewhere (pinned, managed or
 * fine-grained memory, a peer's) sums without parts.
 *
 * Preconditions (else FASTVR_ERR_INVALID_ARGUMENT unless noted):
 *  - q, k, v, dout, o, dq, dk, dv non-NULL and 16-byte aligned (q, dout, o, dq
 *    may be NULL when Nq = 0); lse and row_stats non-NULL and 4-byte aligned
 *    when Nq > 0;
 *  - dq, dk, dv and row_stats overlap no argument;
 *  - size, offset, window and scale rules of fastvr_chunk_attn_fwd, and
 *    H * d < 2^22 (else FASTVR_ERR_UNSUPPORTED).
 * B, H or Nkv equal to 0 (then Nq must be 0): FASTVR_OK, nothing enqueued.
 * Nq = 0 with Nkv > 0 sets dk and dv to zero.
 */
fastvr_status fastvr_chunk_attn_bwd(const void* q, const void* k, const void* v, const float* o, const float* lse,
                                    const void* dout, float* dq, float* dk, float* dv, float* row_stats, int64_t B,
                                    int64_t H, int64_t Nq, int64_t Nkv, int64_t d, int64_t chunk_len,
                                    int64_t q_chunk_offset, int64_t window_chunks, float scale, void* stream);

/*
 * fastvr_chunk_attn_bwd without the row_stats workspace argument, for callers
 * that cannot allocate device memory (code under HIP graph capture, tight
 * serving or training loops, harnesses that forbid allocation).  The row
 * statistics go to a static array of the library instead, 32 MiB
 * (FASTVR_BWD_NOALLOC_MAX_FLOATS floats) that each device holds from the first
 * call until the process ends; the call itself allocates nothing (no hipMalloc,
 * no allocating library routine).  The caller still passes every input and
 * output, with the same meaning, layout and preconditions as in
 * fastvr_chunk_attn_bwd; outputs are identical bit for bit.
 *
 * Limit: 2 * B * H * Nq <= FASTVR_BWD_NOALLOC_MAX_FLOATS, else
 * FASTVR_ERR_UNSUPPORTED (the 1080p sequence needs 1.6 M floats, the 24-head
 * sliding-window sequence 6.7 M).  Every call on one device shares the array:
 * calls that may overlap in time on the same device (different streams or host
 * threads) race and must be serialised by the caller.  FASTVR_ERR_HIP if the
 * array's device address cannot be obtained.
 */
#define FASTVR_BWD_NOALLOC_MAX_FLOATS (8 * 1024 * 1024)
fastvr_status fastvr_chunk_attn_bwd_noalloc(const void* q, const void* k, const void* v, const float* o,
                                            const float* lse, const void* dout, float* dq, float* dk, float* dv,
                                            int64_t B, int64_t H, int64_t Nq, int64_t Nkv, int64_t d,
                                            int64_t chunk_len, int64_t q_chunk_offset, int64_t window_chunks,
                                            float scale, void* stream);

/*
 * One-step latent update (Sec. 3.2, Eq. 9, the update used at inference, Sec.
 * 4.1): z_hat = z_lq - sigma * v, element by element over n elements.
 *
 *   z_lq    bf16 [n]   the LQ latent z_LQ (any layout; v and z_hat share it)
 *   v       bf16 [n]   the velocity the DiT predicts at (z_LQ, tau)
 *   z_hat   fp32 [n] (out_bf16 = 0) or bf16 [n] (out_bf16 = 1)   output
 *   sigma   sigma_tau, the noise level of the starting timestep tau
 * Each element is fma(-sigma, v, z_lq) in fp32 (the exact value rounded once);
 * with out_bf16 = 1 that value is rounded to bf16 (nearest even).
 *
 * Preconditions (else FASTVR_ERR_INVALID_ARGUMENT): n >= 0; pointers non-NULL
 * and 16-byte aligned; sigma finite; out_bf16 in {0, 1}; z_hat overlaps neither
 * input, except that with out_bf16 = 1 it may be exactly z_lq or v (in place).
 * n = 0: FASTVR_OK, nothing enqueued.
 */
fastvr_status fastvr_one_step_update(const void* z_lq, const void* v, void* z_hat, int64_t n, float sigma,
                                     int32_t out_bf16, void* stream);

/*
 * Spatial tiles for tiled inference (Sec. 3 overview: one DiT pass per temporal
 * chunk and spatial tile; Sec. 4.1, Inference: overlapping 64 x 64 latent tiles).
 * The paper does not state the overlap, the placement or the blend; this library
 * takes the following, for fields laid out channels-last x[b, t, y, x, c] over a
 * grid of Hg x Wg positions and T frames (tiles span every frame and cut both
 * spatial axes the same way):
 *  - along an axis of `size` positions: tile length L = min(tile, size);
 *    n = 1 if size <= tile, else ceil((size - overlap) / (tile - overlap)) tiles
 *    at origins a_k = (k (size - L) + (n - 1) / 2) / (n - 1) (integer division):
 *    evenly spaced, a_0 = 0, a_{n-1} = size - L, neighbours overlapping by at
 *    least `overlap`;
 *  - tile (ty, tx) has index ty * nx + tx; a tile tensor is
 *    [B, ny * nx, T, Ly, Lx, C], so a tile batch feeds fastvr_chunk_attn_fwd
 *    directly (batch B * ny * nx, Nq = T * Ly * Lx tokens, chunk_len =
 *    frames per chunk * Ly * Lx);
 *  - blend: position i of a tile has the axis weight min(i + 1, L - i, R),
 *    R = max(overlap, 1); a tile's weight is the product of its two axis
 *    weights, and the blended value is the weight-normalised sum over the tiles
 *    that cover the position (fp32, tiles in index order).
 * Common preconditions (else FASTVR_ERR_INVALID_ARGUMENT unless noted): sizes
 * >= 0; tile >= 1 and 0 <= overlap < tile; tile <= 4096 (else
 * FASTVR_ERR_UNSUPPORTED); Wg * C < 2^31 (else FASTVR_ERR_UNSUPPORTED); tensors
 * contiguous, pointers 16-byte aligned (z_lq: 8-byte); outputs overlap no
 * input.  An empty field (any size 0): FASTVR_OK, nothing enqueued.
 */

/* Host only: number of tiles and tile length along one axis of `size` >= 1. */
fastvr_status fastvr_tile_axis(int64_t size, int64_t tile, int64_t overlap, int64_t* n_tiles, int64_t* tile_len);

/* tiles bf16 [B, ny*nx, T, Ly, Lx, C] <- x bf16 [B, T, Hg, Wg, C]; C a multiple of 8. */
fastvr_status fastvr_tile_gather(const void* x, void* tiles, int64_t B, int64_t T, int64_t Hg, int64_t Wg, int64_t C,
                                 int64_t tile, int64_t overlap, void* stream);

/* out fp32 [B, T, Hg, Wg, C] <- blend of tiles fp32 [B, ny*nx, T, Ly, Lx, C]; C a multiple of 4. */
fastvr_status fastvr_tile_blend(const float* tiles, float* out, int64_t B, int64_t T, int64_t Hg, int64_t Wg,
                                int64_t C, int64_t tile, int64_t overlap, void* stream);

/* The blend fused with the one-step update of Eq. 9 (Sec. 3.2):
 * z_hat fp32 [B, T, Hg, Wg, C] = z_lq - sigma * blend(v_tiles), z_lq bf16 of the
 * same shape (each element fma(-sigma, blend, z) in fp32); sigma finite. */
fastvr_status fastvr_tile_blend_update(const float* v_tiles, const void* z_lq, float* z_hat, float sigma, int64_t B,
                                       int64_t T, int64_t Hg, int64_t Wg, int64_t C, int64_t tile, int64_t overlap,
                                       void* stream);

/*
 * Rotary positions of query or key heads, and their gradient.  In each head the
 * first 2 * n_pairs elements are n_pairs points of the plane, the others pass
 * unchanged.  Pair p turns by the angle position[axis(p)] * inv_freq[p]:
 *   (a, b)  ->  amplitude * (a cos - b sin, a sin + b cos)
 * with (a, b) = elements (2p, 2p + 1) when interleaved, (p, p + n_pairs)
 * otherwise.  inverse = 1 turns by the negative angle, with the same amplitude: the
 * gradient of the call with inverse = 0.  Angles are taken in fp64 (and must stay
 * below 2^51 radians), the products in fp32.
 *
 *   x          bf16 (x_fp32 = 0) or fp32 [B, N, H, d] view   input
 *   y          bf16 (y_fp32 = 0) or fp32 [B, N, H, d] view   output, fully overwritten
 *   positions  int32 [B, N, n_axes] (batch stride pos_sb, 0: shared)   position of each token
 *   inv_freq   fp64 [n_pairs]                                radians per position
 * Pairs p < split1 turn with axis 0, split1 <= p < split2 with axis 1, the others
 * with axis 2 (a frame, row and column of a video token, say); axes that do not
 * exist own no pairs: split1 = n_pairs for one axis, split2 = n_pairs for two.
 *
 * Preconditions (else FASTVR_ERR_INVALID_ARGUMENT unless noted): sizes >= 0; d in
 * {64, 128}, B and H <= 65535, N <= 2^24 (else FASTVR_ERR_UNSUPPORTED);
 * 0 <= n_pairs <= d / 2; 1 <= n_axes <= 3; 0 <= split1 <= split2 <= n_pairs as above;
 * view rules of fastvr_chunk_attn_fwd_ex for x and y; positions 4-byte and
 * inv_freq 8-byte aligned, non-NULL (inv_freq may be NULL when n_pairs = 0);
 * pos_sb = 0 or >= N * n_axes; amplitude finite; y overlaps no input, except that
 * it may be exactly x (same pointer, type and strides): in place.
 * B, N or H equal to 0: FASTVR_OK, nothing enqueued.
 */
fastvr_status fastvr_rope(const void* x, int64_t x_sb, int64_t x_st, int32_t x_fp32, void* y, int64_t y_sb,
                          int64_t y_st, int32_t y_fp32, const int32_t* positions, int64_t pos_sb, int64_t n_axes,
                          int64_t split1, int64_t split2, const double* inv_freq, int64_t n_pairs, double amplitude,
                          int32_t interleaved, int32_t inverse, int64_t B, int64_t N, int64_t H, int64_t d,
                          void* stream);

/*
 * KV cache in 4 bits: microscaled e2m1 elements (values 0, 0.5, 1, 1.5, 2, 3, 4, 6
 * and their negatives) with one power-of-two scale for 32 elements along head_dim,
 * 0.53 instead of 2 bytes an element.  The cache is four tensors, head by head
 * (a head's tokens are contiguous):
 *   k_codes,  v_codes   uint8 [B, H, capacity, d / 2]    element 2i in the low half of byte i
 *   k_scales, v_scales  uint8 [B, H, capacity, d / 32]   scale 2^(byte - 127), 2 <= byte <= 252; 255: NaN
 * A block's scale 2^e is the one that puts its largest magnitude a into
 * [3.5, 7) 2^e (-125 <= e <= 125), so that a goes to the nearest of 4 2^e and 6 2^e;
 * each element goes to the nearest value, ties to the even code.  A block that holds an
 * infinity or NaN stands for NaN (byte 255, codes 0).  The values that codes and
 * scales stand for are exact in bf16.
 * Zeros, as of a new cache, stand for zeros.  What other blocks with byte 0 or 1, or any
 * with 253 or 254, stand for is undefined to the calls that see them; append writes none.
 *
 * fastvr_kv4_append: n_new rows of K and V (bf16 [B, n_new, H, d] views) go to
 * token rows first .. first + n_new - 1 of every sequence, or, when starts (int32
 * [B], device memory) is given, to rows starts[b] + 0 .. n_new - 1 of sequence b
 * (first is not used then); of these, rows outside 0 .. capacity - 1 are dropped.
 * All other rows are left as they are.
 * fastvr_kv4_read: the values of n token rows, first or starts as above, as bf16
 * [B, n, H, d] views; with starts, rows outside the cache read as zero.
 *
 * Preconditions (else FASTVR_ERR_INVALID_ARGUMENT unless noted): sizes >= 0; d in
 * {64, 128}, B <= 32767, H <= 65535, capacity <= FASTVR_KV4_MAX_CAPACITY (else
 * FASTVR_ERR_UNSUPPORTED); without starts, first >= 0 and first + n <= capacity
 * (else FASTVR_ERR_CAPACITY); cache tensors contiguous, 16-byte aligned, and
 * overlapping nothing; view rules of fastvr_chunk_attn_fwd_ex for the bf16 tensors;
 * outputs overlap nothing; starts NULL or 4-byte aligned.
 * B, H, n_new or n equal to 0: FASTVR_OK, nothing enqueued.
 */
#define FASTVR_KV4_MAX_CAPACITY (16 * 1024 * 1024)
fastvr_status fastvr_kv4_append(void* k_codes, void* k_scales, void* v_codes, void* v_scales, const void* k_new,
                                int64_t k_sb, int64_t k_st, const void* v_new, int64_t v_sb, int64_t v_st,
                                const int32_t* starts, int64_t B, int64_t H, int64_t d, int64_t capacity,
                                int64_t first, int64_t n_new, void* stream);
fastvr_status fastvr_kv4_read(const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales,
                              void* k_out, int64_t k_sb, int64_t k_st, void* v_out, int64_t v_sb, int64_t v_st,
                              const int32_t* starts, int64_t B, int64_t H, int64_t d, int64_t capacity, int64_t first,
                              int64_t n, void* stream);

/*
 * Chunk-causal attention of the newest tokens over a 4-bit cache: from one token
 * of each sequence (serving) to whole chunks (streaming).  Sequence b holds
 * len_b = cache_len tokens or, when lens (int32 [B], device memory) is given,
 * len_b = min(max(lens[b], 0), cache_len).  Query row i is the token at position
 * P = len_b - Nq + i, which lies in chunk c = P / chunk_len and sees the keys
 *   max(0, c - window_chunks) * chunk_len .. min((c + 1) * chunk_len, len_b) - 1
 * (window_chunks = -1: from 0).  chunk_len >= cache_len: every row sees the whole
 * cache; chunk_len = 1: token-causal, window_chunks = w - 1 a sliding window of w
 * tokens.  Rows with P < 0 (padding in front of a short sequence) see nothing:
 * O = 0 and LSE = -infinity.  H query heads share Hkv key heads in order:
 * query head h reads key head h / (H / Hkv).  A key that a row does not see has no
 * effect on it, whatever it stands for.
 *
 *   q    bf16 [B, Nq, H, d] view
 *   o    fp32 (o_bf16 = 0) or bf16 [B, Nq, H, d] view, fully overwritten
 *   lse  fp32 [B, H, Nq] contiguous, or NULL
 *   workspace  16-byte aligned device memory of workspace_bytes >= what
 *              fastvr_kv4_attn_workspace gives for these sizes (may be NULL for 0);
 *              the call's own until its work on `stream` has ended
 * Results do not depend on the workspace's contents; equal calls give equal bits.
 * Scores, LSE and all sums are fp32; the softmax weights are held to 2^-16 of themselves
 * where o is fp32, and may be rounded to bf16 (to 2^-8) where o is.  The scores of keys that a
 * row sees stay below 2e38 in magnitude (fp32's range, in base 2).
 *
 * Preconditions (else FASTVR_ERR_INVALID_ARGUMENT unless noted): sizes >= 0; d in
 * {64, 128}; H a multiple of Hkv; 0 <= cache_len <= capacity; chunk_len >= 1;
 * window_chunks >= -1; scale finite; cache tensors contiguous, 16-byte aligned; view
 * rules of fastvr_chunk_attn_fwd_ex for q and o; lens NULL or 4-byte aligned; o,
 * lse and workspace overlap nothing; capacity <= FASTVR_KV4_MAX_CAPACITY, H <= 65535,
 * Nq * H and token strides below 2^31 and not more work items than one launch holds
 * (else FASTVR_ERR_UNSUPPORTED).
 * B, H or Nq equal to 0: FASTVR_OK, nothing enqueued.
 */
fastvr_status fastvr_kv4_attn_workspace(int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t d, int64_t cache_len,
                                        int64_t chunk_len, int64_t window_chunks, int64_t* bytes);
fastvr_status fastvr_kv4_attn(const void* q, int64_t q_sb, int64_t q_st, const void* k_codes, const void* k_scales,
                              const void* v_codes, const void* v_scales, void* o, int64_t o_sb, int64_t o_st,
                              int32_t o_bf16, float* lse, void* workspace, int64_t workspace_bytes,
                              const int32_t* lens, int64_t B, int64_t H, int64_t Hkv, int64_t Nq, int64_t d,
                              int64_t capacity, int64_t cache_len, int64_t chunk_len, int64_t window_chunks,
                              float scale, void* stream);

/* Static string naming a status code ("FASTVR_OK", ...); never NULL. */
const char* fastvr_status_string(fastvr_status s);

/* Detail of the last failing call on this thread ("" if none).  The pointer is
   valid until the next library call on the same thread. */
const char* fastvr_last_error(void);

/* FASTVR_ABI_VERSION of the built library. */
int fastvr_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* FASTVR_H */
