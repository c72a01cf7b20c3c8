/*
 * hf.h -- C ABI of libhf: hybrid attention for an autoregressive streaming video denoiser
 * (block-sparse sliding-window attention over a rolling KV cache + linear-attention history state).
 *
 * One hf_ctx lives on ONE CUDA device and owns, per layer: the rolling cache of the last
 * P = window_frames/chunk_frames - 1 clean chunks (K, V, pooled K), the linear state
 * S [B,H,d,d] / z [B,H,d] in fp32, the merge projection, the last block selection and scratch.
 * The caller owns q/k/v/o.  Unless a parameter says "host", every data pointer is a DEVICE pointer
 * on the context's device, 16-byte aligned, to a contiguous tensor laid out [B, H, T, d] (d fastest)
 * of bf16.  `stream` is a cudaStream_t passed as void* (NULL = the default stream).  Calls enqueue
 * work on `stream` and return; only create / destroy / the *_host calls / hf_get_device_status
 * synchronise.  Every call returns an hf_status; an invalid argument never launches a kernel.
 * Nothing here throws, aborts or traps the device.
 *
 * Concurrency: ONE stream per context at a time.  The scratch buffers (pooled means, split partial sums, the history
 * term of the two-kernel forward path, the staging buffers of the *_host calls), the side stream and its two events
 * belong to the context, not to a layer: two calls on the same context whose work may overlap on the device -- two
 * streams, or two host threads -- race on them, even for different layers.  Calls on one stream, in any order of layers,
 * are safe; so are different contexts on different streams.  To change streams, synchronise the old one first.
 *
 * Logical key-block order seen by selection and attention: oldest cached chunk first, newest cached
 * chunk, then the current chunk.  Every chunk is cut into blocks of `block` tokens from its own first
 * token; a short last block is legal (its mean uses its own length).
 */
#ifndef HF_H_
#define HF_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hf_ctx hf_ctx;

typedef enum {
    HF_OK = 0,
    HF_ERR_INVALID_ARG = 1,   /* null / misaligned pointer, bad layer index                   */
    HF_ERR_SHAPE = 2,         /* configuration or size outside what the kernels support       */
    HF_ERR_STATE = 3,         /* call order: e.g. attention with no selection available       */
    HF_ERR_UNSUPPORTED = 4,
    HF_ERR_NOMEM = 5,
    HF_ERR_CUDA = 6,          /* a CUDA runtime call failed (no device, launch error, ...)    */
    HF_ERR_DEVICE_TIMEOUT = 7 /* a bounded device-side wait ran out; see hf_get_device_status */
} hf_status;

enum { HF_PHI_ELU1 = 0 };                                /* phi(x) = elu(x) + 1                 */
enum { HF_MERGE_IDENTITY = 0, HF_MERGE_PER_HEAD = 1, HF_MERGE_FULL_WIDTH = 2 };   /* "Linear" of Eq. 4: none | W[H,d,d] | W[H d, H d] */
enum { HF_SWA_AUTO = 0, HF_SWA_MMA = 1, HF_SWA_TCGEN05 = 2, HF_SWA_TCGEN05_PINGPONG = 3 }; /* sparse-attention kernel choice */
enum { HF_Z_SUM = 0, HF_Z_FRAME_MEAN = 1 };              /* z of Eq. 3: sum of phi(K) rows | per-frame means */

typedef struct {
    int batch, heads, head_dim;      /* head_dim d in {64, 128}                                         */
    int tokens_per_frame;            /* tokens of one latent frame                                      */
    int chunk_frames;                /* latent frames per chunk; T_c = tokens_per_frame * chunk_frames  */
    int window_frames;               /* sliding window w in frames, counts the current chunk;
                                        a multiple of chunk_frames, at most 8 chunks                    */
    int block;                       /* b_q = b_kv in {16, 64, 128}                                     */
    int topk;                        /* > 0: key blocks kept per query block                            */
    int keep_permille;               /* used when topk == 0: k = ceil(keep_permille * T_n / 1000)       */
    int layers;                      /* independent layer states held by the context                    */
    int phi;                         /* HF_PHI_ELU1                                                     */
    float eps;                       /* added to the denominator phi(q).z of Eq. 4                      */
    int merge;                       /* HF_MERGE_IDENTITY | HF_MERGE_PER_HEAD | HF_MERGE_FULL_WIDTH     */
    int swa_kernel;                  /* HF_SWA_AUTO | HF_SWA_MMA | HF_SWA_TCGEN05 | HF_SWA_TCGEN05_PINGPONG */
    int z_mode;                      /* HF_Z_SUM: z += sum_t phi(K_ev[t]) (default).  HF_Z_FRAME_MEAN: Eq. 3 as printed,
                                        z += sum over evicted latent frames of the mean of phi(K) over the frame's
                                        tokens; absorbed token counts must then be multiples of tokens_per_frame      */
    int sink_frames;                 /* latent frames at the start of the stream kept visible for ever (attention sink):
                                        a multiple of chunk_frames; those first chunks go to slots of their own, as the oldest
                                        logical key blocks, and are never evicted nor folded into the state.  Sink chunks +
                                        window chunks may not exceed 8                                                   */
} hf_config;

/* Fields of hf_query(). */
enum {
    HF_Q_CACHED_CHUNKS = 0,   /* clean chunks now in the rolling cache of the layer (sink chunks not counted) */
    HF_Q_KEY_BLOCKS = 1,      /* T_n a forward would see now: (sink + cached + 1) * blocks per chunk   */
    HF_Q_KEPT_BLOCKS = 2,     /* k_eff = min(k, T_n) for that T_n                                      */
    HF_Q_ABSORBED_TOKENS = 3, /* tokens folded into (S, z) so far (per batch*head)                     */
    HF_Q_QUERY_BLOCKS = 4,    /* T_m = ceil(T_c / block)                                               */
    HF_Q_MASK_WORDS = 5,      /* uint32 words per mask row = ceil(max T_n / 32)                        */
    HF_Q_SWA_KERNEL = 6,      /* kernel hf_sparse_swa resolves to (HF_SWA_MMA | HF_SWA_TCGEN05 | ..._PINGPONG) */
    HF_Q_SINK_CHUNKS = 7      /* sink chunks held so far                                               */
};

/* Create a context on CUDA device `device` (allocates all persistent buffers, zero state).
 * Errors: HF_ERR_INVALID_ARG (null), HF_ERR_SHAPE (unsupported sizes), HF_ERR_CUDA, HF_ERR_NOMEM. */
hf_status hf_create(const hf_config* cfg, int device, hf_ctx** out);
hf_status hf_destroy(hf_ctx* ctx);

/* Empty the rolling cache and zero (S, z) of one layer (layer = -1: all layers). */
hf_status hf_reset(hf_ctx* ctx, int layer, void* stream);

/* Merge projection of the history branch ("Linear" in Eq. 4; the paper does not give its shape).
 *   HF_MERGE_PER_HEAD (default reading): one d x d matrix per head, y = W_h h + bias_h.  W: bf16 [H, d, d] row-major
 *     (row = output dim), bias: bf16 [H, d] or NULL.  The matrix is folded into the state (S W_h^T), so it costs nothing
 *     per call.
 *   HF_MERGE_FULL_WIDTH: one matrix over the model width, y = W x + bias with x = the read-outs of all heads side by
 *     side (head-major).  W: bf16 [H d, H d] row-major (row = output feature), bias: bf16 [H d] or NULL.  It couples the
 *     heads: the read-out kernel is followed by a projection kernel, and the attention kernel adds the result.
 * Copied into the context.  HF_ERR_STATE if the context was created with HF_MERGE_IDENTITY. */
hf_status hf_set_merge_weights(hf_ctx* ctx, int layer, const void* W, const void* bias, void* stream);

/* Rotation inside the linear branch (Eq. 3: RoPE(phi(K))^T V in the state; Eq. 4: RoPE(phi(Q)) in the numerator only, the
 * normaliser never rotates).  The rotation acts on feature pairs (2i, 2i+1); the angles are the caller's: device float
 * tables cos / sin [T_c, d/2], one row per token of a chunk, shared by batch, heads and layers (e.g. built from the
 * capped relative temporal index of Eq. 8 and the spatial coordinates).  cos_q / sin_q rotate the queries of every later
 * hf_linear_attn / hf_hybrid_forward; cos_k / sin_k rotate the keys of every chunk folded into the state from now on
 * (they are applied when the chunk is absorbed).  The tables are copied into the context.  A NULL pair switches that
 * rotation off (the default).  With key tables set, hf_state_absorb accepts at most T_c tokens per call. */
hf_status hf_set_rope(hf_ctx* ctx, const float* cos_q, const float* sin_q, const float* cos_k, const float* sin_k, void* stream);

/* Relative temporal RoPE of the softmax branch (Sec. 3.3, Eq. 8): the temporal index of the chunk being generated counts
 * up with the stream until it reaches t0 (21 in the paper) and stays there; the keys in the cache are re-indexed by their
 * offset to the current chunk.  With this set, q and k are passed to every call WITHOUT temporal rotation (their spatial
 * rotation is the caller's and never changes); the library turns feature pairs [first_pair, first_pair + n_pairs) -- pair p
 * = features (2p, 2p+1) -- of every token by (index of its frame) x (frequency of the pair):
 *   - the queries and the current chunk's keys of a forward call to Eq. 8's indices (the stream position is the number of
 *     frames committed to that layer so far), in the pooling pass that the selection needs anyway; both branches see the
 *     rotated queries;
 *   - a committed chunk's keys to the indices they have while the NEXT chunk is generated; once the cap is reached every
 *     commit turns the chunks that stay in the window back by chunk_frames index steps, in place (keys and block means);
 *     the chunk that leaves is folded into the state as the window last saw it; sink chunks keep their own indices.
 * The cache stores bf16, so each turn rounds once more (at most window/chunk roundings in a key's life).
 *   cos_tab, sin_tab   device float [t0 + 1, n_pairs]: cosine and sine of (index steps) x (frequency of the pair); copied.
 * Must be set while no chunk has been committed (HF_ERR_STATE otherwise); both tables NULL switches it off.
 * The order of the float32 operations of a turn is fixed (the rotated values decide the block selection): x0' = x0 c - x1 s,
 * x1' = x0 s + x1 c, products and sums rounded separately, result rounded to bf16. */
hf_status hf_set_temporal_rope(hf_ctx* ctx, int t0, int first_pair, int n_pairs, const float* cos_tab, const float* sin_tab,
                               void* stream);

/* Alg. 2, cache commit of a clean chunk: k, v bf16 [B,H,T_c,d].  If the cache already holds P chunks the oldest
 * is folded into the state (Eq. 3: S += phi(K_ev)^T V_ev, z += sum phi(K_ev)) and leaves the window; the chunk's
 * K, V are copied in and its per-block K means stored.  The ring has P + 1 slots per layer (a spare one), so the copy
 * of the new chunk and the state update of the old one run side by side; when the call's work is done in stream order
 * both have happened, and the evicted chunk's slot is not written before the next commit.  With P = 0 the chunk goes
 * straight into the state and nothing is cached.  Device memory per layer: (P + 1 + sink chunks) x 2 x B*H*T_c*d bf16. */
hf_status hf_kv_append(hf_ctx* ctx, int layer, const void* k, const void* v, void* stream);

/* Eq. 3 on caller-supplied tokens: k_ev, v_ev bf16 [B,H,n_tokens,d], any n_tokens >= 1. */
hf_status hf_state_absorb(hf_ctx* ctx, int layer, const void* k_ev, const void* v_ev, int n_tokens, void* stream);

/* Alg. 2's cache commit for layers first_layer .. first_layer + n_layers - 1 in one call.  In the sampler every layer
 * commits its clean chunk at the same moment ("if KV full: pop(0) -> update LN; KV.append", once per chunk), and one
 * layer's 28.75 MB at the 832x480 shape is too small a launch to use the memory system; here the chunks that leave are
 * folded into their layers' states by ONE persistent launch (Eq. 3; a thread block owns a (layer, batch*head) state for
 * the whole token range, so there are no partial sums and no second kernel to add them) and the new chunks are copied in
 * and pooled by one more.
 *   k, v   HOST arrays of n_layers DEVICE pointers, bf16 [B,H,T_c,d] each (entry l belongs to layer first_layer + l)
 * Every layer ends up exactly as after hf_kv_append(layer, k[l], v[l]): same cache contents and the same bits in S and
 * z (the token range is cut and summed in the same order).  Layers of the call that are in different phases of the
 * protocol (some still filling the window, some evicting), a window of one chunk, the temporal rotation, or two layers of
 * few heads and long chunks, whose state updates fill the device better one after the other, are handled layer by layer
 * inside the call.  A state update of more (layer, batch*head) pairs than the device has SMs grows its scratch (and waits for
 * the stream) when no call of that size came before: capture such a call into a graph only after the largest one. */
hf_status hf_kv_append_layers(hf_ctx* ctx, int first_layer, int n_layers, const void* const* k, const void* const* v, void* stream);

/* Eq. 3 on caller-supplied tokens for several layers at once: k_ev, v_ev device bf16 [n_layers, B, H, n_tokens, d]
 * (slice l goes into the state of layer first_layer + l).  Same result, bit for bit, as n_layers calls of
 * hf_state_absorb. */
hf_status hf_state_absorb_layers(hf_ctx* ctx, int first_layer, int n_layers, const void* k_ev, const void* v_ev, int n_tokens,
                                 void* stream);

/* Eq. 5 + top-K rule (Alg. 3: M_c[i,j] = 1 iff block j is among the K best of row i): block means of q and of
 * the window's keys (cached chunks + k_cur), scores in a fixed float32 operation order, per (batch, head, query
 * block) the k_eff highest scores kept, equal scores going to the lower block index.  The selection is kept in
 * the context for hf_sparse_swa and optionally written out:
 *   mask_out   uint32 [B,H,T_m,HF_Q_MASK_WORDS], bit (j & 31) of word (j >> 5) = block j kept;  or NULL
 *   idx_out    int32  [B,H,T_m,k_eff] kept block indices ascending;                            or NULL
 *   scores_out float  [B,H,T_m,T_n] raw scores A_ij;                                           or NULL */
hf_status hf_block_select(hf_ctx* ctx, int layer, const void* q, const void* k_cur,
                          uint32_t* mask_out, int32_t* idx_out, float* scores_out, void* stream);

/* Eq. 6 / Alg. 3 inner loops: o_local[r] = softmax_c(q_r . k_c / sqrt(d)) V over the tokens c of the kept key
 * blocks of r's query block.  idx: int32 [B,H,T_m,k_eff] ascending block indices, or NULL = the context's last
 * selection for this layer (HF_ERR_STATE if none or if the cache changed since).  o_local: bf16 [B,H,T_c,d].
 * lse: float [B,H,T_c] natural-log sum of exp of the scaled logits, or NULL.
 * The list lives on the device, so the host cannot look at it: the kernel checks every entry against [0, T_n), reads
 * block 0 in place of an entry outside it (no address is ever formed from such an entry) and sets flag 2 of the
 * device status word; the rows of that query block are then meaningless and hf_get_device_status reports
 * HF_ERR_INVALID_ARG. */
hf_status hf_sparse_swa(hf_ctx* ctx, int layer, const void* q, const void* k_cur, const void* v_cur,
                        const int32_t* idx, void* o_local, float* lse, void* stream);

/* Gradient of Eq. 6 with respect to the queries: the first piece of the backward pass that the training rollout needs
 * for the denoising step it runs with gradient (Alg. 1).  With p = softmax over the kept keys and g = dL/dO_local,
 *   dq_r = (1 / sqrt(d)) sum_c p_rc (g_r . v_c - g_r . o_local_r) k_c      (the block mask is the forward's, held fixed)
 *   q, k_cur, v_cur, idx   as for hf_sparse_swa (same cache contents, same selection)
 *   o_local bf16 [B,H,T_c,d], lse float [B,H,T_c]   what hf_sparse_swa returned for them
 *   d_o bf16 [B,H,T_c,d] = dL/dO_local;  dq bf16 [B,H,T_c,d] out
 * 128-token blocks only (HF_ERR_UNSUPPORTED otherwise, and with the temporal rotation set).  The history branch's share of
 * dq comes from hf_linear_attn_backward_dq. */
hf_status hf_sparse_swa_backward_dq(hf_ctx* ctx, int layer, const void* q, const void* k_cur, const void* v_cur, const int32_t* idx,
                                    const void* o_local, const float* lse, const void* d_o, void* dq, void* stream);

/* Gradients of Eq. 6 with respect to the CURRENT chunk's keys and values (the cached chunks come from earlier,
 * gradient-free passes of the rollout and receive none): with the notation above, for key token c of the current chunk
 *   dv_c = sum_r p_rc g_r,     dk_c = (1 / sqrt(d)) sum_r p_rc (g_r . v_c - g_r . o_local_r) q_r
 * over the query rows r whose query block keeps c's key block -- the context's last selection for this layer
 * (hf_block_select or hf_hybrid_forward; HF_ERR_STATE if the cache changed since).  Arguments as for
 * hf_sparse_swa_backward_dq; dk, dv bf16 [B,H,T_c,d] out (zero for a key block that no query block keeps). */
hf_status hf_sparse_swa_backward_dkv(hf_ctx* ctx, int layer, const void* q, const void* k_cur, const void* v_cur, const void* o_local,
                                     const float* lse, const void* d_o, void* dk, void* dv, void* stream);

/* Gradient of Eq. 4 (hf_linear_attn, per-head or identity merge, no rotation) with respect to the queries.  With
 * f = phi(q_r), den = f . z + eps, S' = S W^T and g_r = d_o[r] (the gradient with respect to o_hist[r], which by Eq. 7 is
 * the gradient with respect to the merged output):
 *   u = S' g_r,   df = (u - (f . u / den) z) / den,   dq[r] = df * phi'(q_r)   (phi' = 1 above zero, e^x otherwise).
 * S, z and the cached chunks come from earlier, gradient-free passes and receive nothing.  The total gradient of the
 * hybrid output with respect to q is this plus hf_sparse_swa_backward_dq's (the caller adds them).  q, d_o bf16
 * [B,H,T_c,d] device; dq bf16 [B,H,T_c,d] out.  HF_ERR_UNSUPPORTED with the full-width merge or a rotation set. */
hf_status hf_linear_attn_backward_dq(hf_ctx* ctx, int layer, const void* q, const void* d_o, void* dq, void* stream);

/* Eq. 4 without rotation: o_hist[r] = W (phi(q_r) S / (phi(q_r) . z + eps)) + bias, bf16 [B,H,T_c,d]. */
hf_status hf_linear_attn(hf_ctx* ctx, int layer, const void* q, void* o_hist, void* stream);

/* Eq. 6 + Eq. 4 + Eq. 7 for a selection that is already made (idx as for hf_sparse_swa; NULL = the context's last
 * selection): o = o_local + o_history, rounded once to bf16 [B,H,T_c,d].  hf_hybrid_forward is hf_block_select followed
 * by this call.  With the tcgen05 attention kernel and the per-head or identity merge, rotated or not, the attention kernel
 * forms the history term on the tensor cores at the end of each unit of 128 query rows (blocks of 16 and 64 tokens: after a
 * small kernel that merges the kept lists of a unit); otherwise the read-out kernel runs first and the attention kernel adds
 * its result. */
hf_status hf_sparse_swa_merged(hf_ctx* ctx, int layer, const void* q, const void* k_cur, const void* v_cur, const int32_t* idx,
                               void* o, void* stream);

/* Alg. 3 + Eq. 7 for one denoising step: selection, sparse attention and history read-out of q against the
 * cache + (k, v), o = o_local + o_history rounded once to bf16 [B,H,T_c,d]. */
hf_status hf_hybrid_forward(hf_ctx* ctx, int layer, const void* q, const void* k, const void* v, void* o, void* stream);

/* Same two calls for HOST buffers (pinned memory recommended): inputs are copied to staging buffers owned by the
 * context, the device path runs, o is copied back, and the call returns after the stream has drained. */
hf_status hf_hybrid_forward_host(hf_ctx* ctx, int layer, const void* q_host, const void* k_host, const void* v_host,
                                 void* o_host, void* stream);
hf_status hf_kv_append_host(hf_ctx* ctx, int layer, const void* k_host, const void* v_host, void* stream);

/* State update without any allocation.  (No counterpart in the paper: it is the arithmetic of hf_state_absorb,
 * offered for callers that cannot allocate.)
 *
 * Who needs it: code that runs where cudaMalloc is off limits -- inside a region whose memory plan is already
 * frozen (a serving loop that pre-sized its pools and must not perturb them), a callback or plugin that is not
 * allowed to touch the allocator or to create an hf_ctx (which allocates at creation), or a host thread that must
 * not take the allocator's implicit device-wide synchronisation.  hf_state_absorb splits the token range over
 * several thread blocks and needs global scratch for their partial sums; here that scratch is a fixed 16 MiB array
 * compiled into the library image, which every device that loads the library holds until the process exits.
 *
 * Computes, on the current device:  S[bh] += phi(k_ev[bh])^T v_ev[bh],  z[bh] += sum_t phi(k_ev[bh][t])
 *   k_ev, v_ev  device bf16 [batch_heads, n_tokens, head_dim], read only
 *   S           device float [batch_heads, head_dim, head_dim], updated in place (caller initialises it)
 *   z           device float [batch_heads, head_dim], updated in place
 * Limits: head_dim in {64, 128}; 1 <= batch_heads <= 1024 and batch_heads * (head_dim^2 + head_dim) * 4 bytes must
 * fit in 16 MiB - 4 KiB (253 batch*heads at head_dim 128, 1008 at head_dim 64); anything larger returns HF_ERR_SHAPE
 * and launches nothing.  All pointers 16-byte aligned (else HF_ERR_INVALID_ARG).
 * The first call on a device looks up the device address of the scratch array and sets a kernel attribute; make
 * that first call outside any stream capture.  No call here uses cudaMalloc, cudaFree or an allocating library routine.
 * All calls on a device share the one array (each call rewrites the part it reads, so nothing has to be cleared): two calls
 * whose kernels may overlap on the GPU -- different streams, or different threads -- race; keep them stream-ordered. */
hf_status hf_state_absorb_noalloc(const void* k_ev, const void* v_ev, int batch_heads, int n_tokens, int head_dim,
                                  float* S, float* z, void* stream);

/* Copy the state out: S float [B,H,d,d] (row = key feature, column = value dim), z float [B,H,d]; either may be NULL. */
hf_status hf_get_state(hf_ctx* ctx, int layer, float* S, float* z, void* stream);

/* Checkpoint of the whole streaming state of the method (the rolling cache and the linear state, which is all the
 * memory the method carries from chunk to chunk -- Sec. 3.3; Alg. 2's KV and LN), for every layer of the context, into
 * ONE host buffer: per layer the sink chunks and the cached clean chunks (K, V and their pooled block sums, oldest
 * first -- the physical rotation of the ring is not kept), S, z and the absorbed-token count.  Merge weights and
 * rotation tables are parameters, not state: they are not in the image.
 *   host_buf == NULL : *bytes receives the size the image would have now; nothing is copied.
 *   host_buf != NULL : *bytes holds the capacity of host_buf on entry and the bytes written on return;
 *                      HF_ERR_SHAPE (and the needed size in *bytes) if the capacity is too small.
 * Synchronises the device.  The image is only meaningful to hf_state_import of this library version. */
hf_status hf_state_export(hf_ctx* ctx, void* host_buf, size_t* bytes);

/* Load an image written by hf_state_export into a context created with the same configuration (every field that
 * fixes a shape or the arithmetic of the state must match: HF_ERR_SHAPE otherwise; HF_ERR_INVALID_ARG for a buffer
 * that is not an image or is cut short).  All layers are replaced; the folded state is rebuilt from S and the merge
 * weights the context holds at that moment (weights set later refold it again).  A stream that continues after the
 * import produces bit-for-bit what the uninterrupted stream produces.  Synchronises the device.  Nothing is changed
 * when the image is rejected. */
hf_status hf_state_import(hf_ctx* ctx, const void* host_buf, size_t bytes);

/* Host-side bookkeeping values (HF_Q_*). */
hf_status hf_query(hf_ctx* ctx, int layer, int what, int64_t* value);

/* Synchronises the device and reports the device status word.  Flag 1: a bounded wait inside a kernel ran out
 * (detail = where), HF_ERR_DEVICE_TIMEOUT.  Flag 2: a caller's index list held a block index outside [0, T_n)
 * (detail = batch*head and query block of the row, as one number), HF_ERR_INVALID_ARG.  In both cases the result of
 * that launch is invalid, the word is cleared and the context stays usable. */
hf_status hf_get_device_status(hf_ctx* ctx, int* flags, int* detail);

/* Alg. 3 keeps a running row maximum m (m_new = max(m, rowmax S)) and rescales l and O by e^{m - m_new}.  The tcgen05
 * attention kernel (HF_SWA_TCGEN05, what HF_SWA_AUTO resolves to) instead fixes a row's reference after the first kept
 * key blocks that it walks (128 keys; softmax does not depend on the reference), which covers rows whose later blocks rise
 * up to about 100 natural-log units above those; a (batch*head, query block) unit with a row beyond that is computed a second time
 * inside the same launch with the running maximum, so o is the softmax of Eq. 6 for every finite input and no status has
 * to be polled.  This call synchronises the device and reports how many units have taken that second pass since the
 * context was created (a diagnostic: such units cost several times a normal one). */
hf_status hf_slow_path_units(hf_ctx* ctx, int64_t* units);

/* Self-test of the failure path all kernels share (no counterpart in the paper).  Every wait inside a kernel is bounded:
 * when its limit runs out the thread block raises flag 1 of the status word and leaves in the ordinary way.  This call
 * launches a one-warp kernel that waits, under a limit of about a millisecond, on a barrier nothing ever arrives on, so
 * the wait runs out by construction; the next hf_get_device_status must then report HF_ERR_DEVICE_TIMEOUT with detail 77
 * and clear the word, and the context must work as before.  Nothing in it can hang or fault the device. */
hf_status hf_selftest_wait_limit(hf_ctx* ctx, void* stream);

/* Number of kernels the library has launched since the context was created. */
hf_status hf_launch_count(hf_ctx* ctx, int64_t* launches);

/* ------------------------------------------------------------------------------------------------------------------
 * The rest of a denoiser block around the attention: layer norm, rotary positions with several axes, the gated
 * feed-forward, each with its backward pass.  (No counterpart in the paper, which takes them from the pretrained model.)
 *
 * These calls need no context.  They run on the CURRENT device, enqueue work on `stream` and return; scratch is the caller's (`workspace`,
 * whose size the *_workspace calls give; 16-byte aligned; it may be used again as soon as the call's work is done in stream order), so calls
 * on different streams with different workspaces are independent.  They may be captured into a graph once one call of the kind has been
 * made on the device.  Strides are in elements.  Sums, means and products are formed in float32 whatever the type; a result is rounded
 * once.  A call of no rows launches nothing, or clears the parameters' gradients.  Gradients are summed in a fixed order: a call repeated
 * gives the same bits.  A bounded wait that runs out, or a position outside its table, is reported by hf_layers_status. */
enum { HF_BF16 = 0, HF_F16 = 1, HF_F32 = 2 };            /* element types */

/* Layer norm over the last axis: mean and rstd = 1 / sqrt(var + eps) of each row, xhat = (x - mean) rstd,
 *   y = xhat (weight_offset + weight_g) + bias_g,   g = row / rows_per_group (0 for every row when rows_per_group is 0).
 * weight, bias: one row of `width` parameters for each group, param_stride elements apart.  rows_per_group > 0 with weight_offset 1 is
 * the modulated norm of a denoiser (a scale and a shift per latent frame, slices of one modulation tensor). */
typedef struct {
    int type;                    /* of x, y, dy, dx: HF_BF16 | HF_F16 | HF_F32                                        */
    int param_type;              /* of weight and bias: `type` or HF_F32                                              */
    int width;                   /* D, 1 .. 16384                                                                     */
    int64_t rows;
    int64_t x_stride, y_stride, dx_stride;     /* between rows of x, of y or dy, of dx; each >= width                 */
    int64_t rows_per_group;      /* 0: one group                                                                      */
    int64_t param_stride;        /* >= width; not read with one group                                                 */
    float weight_offset;         /* added to weight; not used without weight                                          */
    float eps;                   /* >= 0                                                                              */
} hf_norm_shape;

/* weight, bias, mean, rstd may be NULL (no factor, no shift; not written).  mean, rstd float [rows].  y may be x.  Pointers are aligned to
 * their element, and rows may start anywhere; rows that all start on 16 bytes, with a width of a multiple of 16 bytes, are the fastest.  Of others
 * the whole 16-byte units that hold a row are read (up to 15 bytes in front of it and behind it, whose values do not matter). */
hf_status hf_layer_norm(const hf_norm_shape* shape, const void* x, const void* weight, const void* bias, void* y, float* mean,
                        float* rstd, void* stream);

/* With gh = dy (weight_offset + weight_g):
 *   dx = rstd (gh - mean(gh) - xhat mean(gh xhat)),  dweight_g = sum of dy xhat over the group's rows,  dbias_g = sum of dy.
 * mean, rstd: what the forward returned.  dweight, dbias float [groups, width], contiguous, written, not added to.  dx, and dweight and
 * dbias, may be NULL (not formed).  dx may be dy or x. */
hf_status hf_layer_norm_workspace(const hf_norm_shape* shape, size_t* bytes);
hf_status hf_layer_norm_backward(const hf_norm_shape* shape, const void* dy, const void* x, const float* mean, const float* rstd,
                                 const void* weight, void* dx, float* dweight, float* dbias, void* workspace, void* stream);

/* Rotary positions with several axes (time, height, width of a video's tokens): the first pairs[0] feature pairs of a head turn by the
 * token's position on axis 0, the next pairs[1] by its position on axis 1, and so on; features behind them are copied.
 * (x0, x1) -> (x0 c - x1 s, x0 s + x1 c); with `inverse` the other way round, which is the backward pass.
 *   cos_tab, sin_tab  device float: axis a's table [extent[a], pairs[a]] behind axis a - 1's
 *   pos               device int32 [batch, tokens, axes], or [tokens, axes] for all batches (pos_batch 0).  A position outside [0, extent[a]) is
 *                     taken as 0 and sets flag 2 of the status word.
 * One launch takes up to three tensors of [batch, tokens, heads, head_dim] elements, features contiguous, other axes with strides of
 * their own: q, k and v between the rows of a fused projection and head-major tensors, in either direction.  A tensor with rotate 0 is copied. */
enum { HF_PAIRS_ADJACENT = 0, HF_PAIRS_HALVES = 1 };     /* pair p = features (2p, 2p+1) | (p, P + p), P = sum of pairs */
typedef struct {
    int type;
    int batch, tokens, head_dim;                         /* head_dim even, 2 .. 1024                                  */
    int axes;                                            /* 1 .. 4                                                    */
    int pairs[4], extent[4];                             /* sum of pairs <= head_dim / 2                              */
    int pairing;                                         /* HF_PAIRS_ADJACENT | HF_PAIRS_HALVES                       */
    int inverse;
    int64_t pos_batch;                                   /* int32 between the positions of two batches; 0: shared     */
} hf_rope_shape;
typedef struct {
    const void* x;                                       /* read                                                      */
    void* y;                                             /* written; may be x with the same strides                   */
    int64_t x_batch, x_token, x_head;                    /* strides of x                                              */
    int64_t y_batch, y_token, y_head;
    int heads;
    int rotate;                                          /* 0: copied                                                 */
} hf_rope_tensor;
hf_status hf_rope_axes(const hf_rope_shape* shape, const hf_rope_tensor* tensors, int n_tensors, const float* cos_tab,
                       const float* sin_tab, const int32_t* pos, void* stream);

/* Norms of q and k, their rotation and the split into heads in one pass.  rows [batch, tokens, (heads + 2 kv_heads) head_dim], a fused projection's: q's
 * heads, then k's, then v's.  With r = 1 / sqrt(mean x^2 + eps), the mean over a head (HF_NORM_OVER_HEAD) or over all of q's (of k's) heads of the
 * token (HF_NORM_OVER_WIDTH):   q = R (x r q_weight),  k = R (x r k_weight),  v as it is;   R as hf_rope_axes turns a head (axes, pairs,
 * extent, pairing, tables and positions as there, a position outside its table too).
 * Squares and their mean are float32: where they overflow (features beyond 1.8e19) results are 0 or not finite.
 *   q_weight  [head_dim], or [heads head_dim] with HF_NORM_OVER_WIDTH (k_weight: kv_heads); NULL: 1
 *   heads     q, k, v [batch, heads or kv_heads, tokens, head_dim], features contiguous, other strides free
 * Pointers are aligned to their element; where all start on 16 bytes, head_dim is a multiple of 8 (and, in halves, the sum of pairs of 4) and
 * strides are multiples of 16 bytes, the call is the fastest. */
enum { HF_NORM_OVER_HEAD = 0, HF_NORM_OVER_WIDTH = 1 };
typedef struct {
    int type, param_type;                                /* of rows and heads; of the weights: `type` or HF_F32       */
    int batch, tokens, head_dim;                         /* head_dim even, 2 .. 256                                   */
    int heads, kv_heads;                                 /* kv_heads <= heads; heads x head_dim, in eights up to a power of two, <= 16384 */
    int axes;                                            /* 1 .. 4                                                    */
    int pairs[4], extent[4];
    int pairing;
    int over;
    float eps;                                           /* >= 0                                                      */
    int64_t pos_batch;
    int64_t rows_batch, rows_token;                      /* strides of rows                                           */
    int64_t grad_batch, grad_token;                      /* of their gradient                                         */
} hf_heads_shape;
typedef struct {
    void* p;                                             /* written; backward: read                                   */
    int64_t batch, token, head;                          /* strides                                                   */
} hf_heads_tensor;
hf_status hf_split_heads_norm_rope(const hf_heads_shape* shape, const void* rows, const void* q_weight, const void* k_weight,
                                   const float* cos_tab, const float* sin_tab, const int32_t* pos, const hf_heads_tensor* heads, void* stream);
/* With g = R^T dq, xh = x r, gw = g q_weight:  drows = r (gw - xh mean(gw xh)) for q, likewise for k, dv for v;  dq_weight = sum of g xh over the
 * tokens (with HF_NORM_OVER_HEAD the heads too).  heads: dq, dk, dv.  The weights' gradients are float, written, and may be NULL. */
hf_status hf_split_heads_norm_rope_workspace(const hf_heads_shape* shape, size_t* bytes);
hf_status hf_split_heads_norm_rope_backward(const hf_heads_shape* shape, const hf_heads_tensor* heads, const void* rows, const void* q_weight,
                                            const void* k_weight, const float* cos_tab, const float* sin_tab, const int32_t* pos, void* drows,
                                            float* dq_weight, float* dk_weight, void* workspace, void* stream);

/* Gated feed-forward:  g = x Wg^T,  u = x Wu^T,  h = act(g) u,  y = h Wd^T.   act: silu(g) = g / (1 + e^-g), or the tanh form of gelu.
 *   x [rows, width], Wg, Wu [hidden, width], Wd [out_width, hidden], y [rows, out_width]: bf16 or f16, weights contiguous.
 *   gate, up [rows, hidden] contiguous: g and u for the backward pass, rounded to the type, or both NULL.
 * h is rounded to the type between the two products (the tensor cores take 16-bit operands), from g and u in float32.  With f16 that also
 * bounds h: act(g) u beyond 65504 becomes infinite, and its row of y infinite or NaN, where float32 would hold it; bf16 has float32's range.
 * width, hidden, out_width: multiples of 8; strides too; pointers 16-byte aligned. */
enum { HF_ACT_SILU = 0, HF_ACT_GELU_TANH = 1, HF_ACT_NONE = 2 };       /* (NONE: hf_linear alone) */
typedef struct {
    int type;                    /* HF_BF16 | HF_F16 */
    int act;
    int64_t rows;                /* up to 2^24       */
    int width, hidden, out_width;                        /* up to 2^17 */
    int64_t x_stride, y_stride;                          /* between rows of x, of y or dy */
} hf_ff_shape;
hf_status hf_gated_ff_workspace(const hf_ff_shape* shape, int backward, size_t* bytes);
hf_status hf_gated_ff(const hf_ff_shape* shape, const void* x, const void* w_gate, const void* w_up, const void* w_down, void* y,
                      void* gate, void* up, void* workspace, void* stream);
/* dh = dy Wd,  dg = dh u act'(g),  du = dh act(g),   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x,  dWd = dy^T h  (h from g and u again;
 * dg, du and h rounded to the type: with f16 dg and du below 6.1e-5 lose bits, and below 3e-8 all of them, so small gradients want a
 * scaled dy, as f16 training has it).  gate, up: what the forward returned.  dx [rows, width], dWg, dWu, dWd: the type, contiguous, written.
 * dx, and the three weights' gradients together, may be NULL (not formed). */
hf_status hf_gated_ff_backward(const hf_ff_shape* shape, const void* dy, const void* x, const void* w_gate, const void* w_up,
                               const void* w_down, const void* gate, const void* up, void* dx, void* dw_gate, void* dw_up,
                               void* dw_down, void* workspace, void* stream);

/* A linear layer with its epilogue:  pre = x W^T + bias,  y = residual + gate_g act(pre),  g = row / rows_per_group (0 for every row when that is 0).
 *   x [rows, width], W [out_width, width] contiguous, y and residual [rows, out_width]: bf16 or f16.  bias [out_width], gate [groups, out_width],
 *   rows gate_stride apart: that type or float (param_type).  bias, gate, residual may be NULL; act HF_ACT_NONE: act(pre) = pre.
 *   pre [rows, out_width] contiguous: for the backward pass, rounded to the type, or NULL.
 * Sums and the epilogue are float32; y is rounded once.  With gate rows_per_group of the latent frame and residual the stream x, this is the end of either
 * half of a denoiser block.  width, out_width, strides: multiples of 8; pointers 16-byte aligned.  y may be the residual, with its stride.
 * workspace may be NULL where hf_linear_workspace says 0 bytes. */
typedef struct {
    int type, param_type;        /* HF_BF16 | HF_F16; of bias and gate: `type` or HF_F32 */
    int act;                     /* HF_ACT_NONE | HF_ACT_SILU | HF_ACT_GELU_TANH         */
    int width, out_width;        /* up to 2^17       */
    int64_t rows;                /* up to 2^24       */
    int64_t x_stride, y_stride, residual_stride;         /* between rows of x, of y or dy, of the residual */
    int64_t rows_per_group, gate_stride;                 /* (gate_stride: not read with one group)         */
} hf_linear_shape;
hf_status hf_linear_workspace(const hf_linear_shape* shape, int backward, size_t* bytes);
hf_status hf_linear(const hf_linear_shape* shape, const void* x, const void* weight, const void* bias, const void* gate, const void* residual,
                    void* y, void* pre, void* workspace, void* stream);
/* dp = dy gate_g act'(pre),  dx = dp W,  dW = dp^T x,  dbias = sum of dp over the rows,  dgate_g = sum of dy act(pre) over the group's rows.  dp is rounded
 * to the type for the two products, and not for the sums (f16: as hf_gated_ff_backward says of dg).  pre: what the forward returned; not read with
 * HF_ACT_NONE and without gate.  dx [rows, width], dweight: the type, contiguous; dbias [out_width], dgate [groups, out_width]: float, contiguous;
 * written, each may be NULL.  (The residual's gradient is dy.)  Of no rows: zeros; with rows_per_group > 0 there are then no rows of dgate. */
hf_status hf_linear_backward(const hf_linear_shape* shape, const void* dy, const void* x, const void* weight, const void* pre, const void* gate,
                             void* dx, void* dweight, float* dbias, float* dgate, void* workspace, void* stream);

/* ------------------------------------------------------------------------------------------------------------------
 * A training step's end: the norm of all gradients, and AdamW, each over many tensors at once.  As the calls above: current device, caller's
 * stream, captured like any other work. */

/* out[0] = the 2-norm of all tensors together; out[1] = min(1, max_norm / out[0]), the factor that brings it to max_norm at most (1 for a norm of
 * 0; NaN where the norm is not finite, which hf_adamw takes as a step to leave out).  Squares are formed in float32, so a value beyond 1.8e19
 * counts as not finite, and one below 2e-23 as 0 (below 1e-19 its square has fewer bits); they are summed in double, in a fixed order.  Tensors are contiguous.  out: device, two floats. */
typedef struct {
    const void* p;
    int64_t n;                   /* elements                */
    int type;                    /* HF_BF16 | HF_F16 | HF_F32 */
} hf_gradient;
hf_status hf_gradient_norm_workspace(int n_tensors, size_t* bytes);
hf_status hf_gradient_norm(const hf_gradient* tensors, int n_tensors, float max_norm, float* out, void* workspace, void* stream);

/* One step of AdamW, t = *step + 1 of each tensor, afterwards counted there:
 *   g = factor grad,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   p = p - lr ((m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps) + weight_decay p)
 * in float32; a bf16 parameter is rounded once, from its float32 master where it has one (the master is what the step starts from; p is then
 * only written).  state_bits 32: m, v float.  8: m e4m3, v e5m2 (one byte an element, values times the scale of their block of 256 elements),
 * scales [ceil(n / 256)][2] float for m and v, rounded up or down at random, up with the probability of what is cut off, by a hash of seed, t
 * and the element's place (256 first_block + its index): give every tensor blocks of its own.  A value that is not finite spoils its block of 256.
 * factor: device float, or NULL (1); where it is not finite the call changes nothing.  lr_at: device float that stands for lr, or NULL, so that a
 * captured step follows a schedule.  Pointers are aligned to their element, scales to 8 bytes; a tensor is the fastest where its float32 parts start on
 * 32 bytes, its bf16 parts on 16 and its states in 8 bits on 8.  A tensor is in a call once; two calls on the same tensors or the same counter must not run at the same time. */
typedef struct {
    int param_type;              /* HF_BF16 | HF_F32                    */
    int grad_type;               /* the parameters' type, or HF_F32     */
    int state_bits;              /* 32 | 8                              */
    uint32_t seed;
    double beta1, beta2;         /* in [0, 1)                           */
    double eps;
    const float* factor;
    int32_t* counter;            /* device, 0 before the first call; left 0 */
} hf_adamw_step;
typedef struct {
    void* p;
    const void* g;
    float* master;               /* of bf16 parameters: NULL for all tensors of the call, or for none */
    void* m;
    void* v;
    float* scales;               /* state_bits 8                        */
    int32_t* step;               /* device: steps taken before (counted for a tensor of no elements too, where it is given) */
    const float* lr_at;
    int64_t n;                   /* elements, up to 2^43                */
    int64_t first_block;
    double lr, weight_decay;
} hf_adamw_tensor;
hf_status hf_adamw(const hf_adamw_step* step, const hf_adamw_tensor* tensors, int n_tensors, void* stream);

/* Synchronises the current device and reports the status word of the calls without a context, as hf_get_device_status does for a
 * context's: flag 1 a bounded wait ran out (HF_ERR_DEVICE_TIMEOUT), flag 2 a position outside its table (HF_ERR_INVALID_ARG).  Clears it. */
hf_status hf_layers_status(int* flags, int* detail);

const char* hf_status_string(hf_status s);
const char* hf_last_error(void);   /* text of the last failure on this thread ("" if none) */

#ifdef __cplusplus
}
#endif
#endif /* HF_H_ */
