/*
 * apack.h -- C ABI of the A-PACK inner-LLM prune step on NVIDIA GB300 (sm_103a).
 *
 * A-PACK (Sec. 3.2, "Inner-LLM Query-Aware Compression"; Algorithm 1, the
 * inner-LLM loop) prunes multimodal tokens inside the decoder: at a pruning
 * layer it scores every cached audio and visual token by the attention it
 * receives from the text query (Eq. inner_score), keeps the top fraction of
 * them (Eq. inner) and drops the rest together with their key-value entries,
 * so that later layers and decoding see a shorter sequence.
 *
 * Conventions shared by every entry point:
 *  - Pointers are DEVICE memory unless the name ends in _h (HOST memory).
 *  - The caller owns every buffer.  The library allocates nothing, keeps no
 *    per-call state, never synchronises inside a step and never traps: every
 *    call returns an apack_status.  All device work is enqueued on `stream`
 *    (a cudaStream_t passed as void*; NULL = legacy default stream).
 *  - bf16 data are passed as untyped pointers to 16-bit storage.
 *  - A packed (ragged) batch of B sequences stores token t of sequence b at
 *    row cu_seqlens[b] + t of every per-token array.
 *  - Arguments are checked on the host before anything is enqueued
 *    (APACK_EINVAL).  Problems only the device can see (modality counts that
 *    disagree with the host counts, a bounded wait that gave up) are written
 *    to an error word in the workspace and read with apack_device_error().
 *  - Calls that share a workspace must be ordered (same stream, or joined).
 */
#ifndef APACK_H
#define APACK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t apack_status;
enum {
  APACK_OK = 0,
  APACK_EINVAL = 1,        /* bad argument (null, size, alignment, shape, ratio) */
  APACK_ECUDA = 2,         /* a CUDA runtime or driver call failed */
  APACK_EWORKSPACE = 3,    /* workspace too small (see apack_workspace_size) */
  APACK_ETIMEOUT = 4,      /* device error word: a bounded wait gave up */
  APACK_EDEVICE = 5,       /* device error word: device data disagree with host counts */
  APACK_EUNSUPPORTED = 6   /* shape outside what this build supports (e.g. head_dim != 128) */
};

/* Per-token modality codes.  S, the set of prunable "cached multimodal
   tokens" of Sec. 3.2, is every token coded AUDIO or VISUAL; OTHER tokens
   (system prompt, text, the query itself) are never scored or dropped. */
enum { APACK_MOD_OTHER = 0, APACK_MOD_AUDIO = 1, APACK_MOD_VISUAL = 2 };

/* Selection segments.  PER_MODALITY takes the top-k separately for the audio
   and the visual tokens of each sequence (two keep counts per sequence);
   JOINT takes one top-k over all of S, the literal form of Eq. inner. */
enum { APACK_SELECT_PER_MODALITY = 0, APACK_SELECT_JOINT = 1 };

/* Softmax domain of the relevance scores (apack_seqs.softmax_domain).
   MM: Eq. inner_score as printed, the denominator runs over the cached
   multimodal tokens S of the sequence only.
   CAUSAL_ROW: the denominator is the decoder's own attention row, every token
   the query row attends to causally (system, text, audio, visual and the
   query tokens up to and including its own position); query row r sits at
   position q_start + r of its sequence (apack_seqs.q_start_h; by default the
   query rows are the last n_q tokens, q_start = len - n_q), and a token of S
   that a row cannot see contributes 0 for that row. */
enum { APACK_SOFTMAX_MM = 0, APACK_SOFTMAX_CAUSAL_ROW = 1 };

/* Maximum sizes of this build. */
#define APACK_HEAD_DIM 128
#define APACK_MAX_SEQS 4096

/* The packed batch entering a pruning layer. */
typedef struct apack_seqs {
  int32_t num_seqs;             /* B, 1 .. APACK_MAX_SEQS */
  const int32_t *cu_seqlens_h;  /* [B+1] token offsets, cu_seqlens_h[0] == 0, non-decreasing */
  const int32_t *cu_qlens_h;    /* [B+1] offsets of each sequence's query rows in the packed Q */
  const int32_t *n_audio_h;     /* [B] audio tokens per sequence (verified on the device) */
  const int32_t *n_visual_h;    /* [B] visual tokens per sequence (verified on the device);
                                   with APACK_SELECT_JOINT only n_audio_h + n_visual_h = |S| is
                                   used, so a caller that knows only |S| may pass (|S|, 0) */
  const uint8_t *modality;      /* [T] APACK_MOD_* per token, T = cu_seqlens_h[B] */
  int32_t num_q_heads;          /* Hq */
  int32_t num_kv_heads;         /* Hkv; Hq % Hkv == 0, query head h reads key head h / (Hq/Hkv) */
  int32_t head_dim;             /* D; must be APACK_HEAD_DIM */
  int32_t softmax_domain;       /* APACK_SOFTMAX_MM (0, zero-initialised default) or
                                   APACK_SOFTMAX_CAUSAL_ROW (needs n_q <= len per sequence) */
  const int32_t *q_start_h;     /* [B] or NULL: position of each sequence's first query row
                                   within the sequence (the query span of Sec. 3.2's problem
                                   statement), 0 <= q_start, q_start + n_q <= len; NULL means
                                   the span ends the sequence.  Read in the CAUSAL_ROW domain
                                   only (in the MM domain no query token is in S). */
} apack_seqs;

/* One group of per-token planes to compact (e.g. the K cache of layers l..L-1).
   Plane p, token row t lives at  base + p*plane_stride + t*row_stride.
   Rows of >= 16 bytes whose addresses and strides are 16-byte aligned take
   the vectorised path; any other row size is copied with narrower accesses.
   src and dst must not overlap unless src == dst with equal strides (in place). */
typedef struct apack_plane {
  const void *src;
  void *dst;
  int64_t src_plane_stride;     /* bytes between planes of src */
  int64_t dst_plane_stride;     /* bytes between planes of dst */
  int64_t src_row_stride;       /* bytes between token rows of src */
  int64_t dst_row_stride;       /* bytes between token rows of dst */
  int64_t row_bytes;            /* bytes copied per token row */
  int32_t num_planes;
  int32_t reserved;
} apack_plane;

/* Bytes of device workspace the calls below need for this batch (256-byte
   aligned start required).  Depends on B, the query rows and head counts.
   Bytes 0..15 are the device error word, bytes 256..1023 belong to the
   in-place compaction of apack_compact; everything else is scratch that the
   scoring writes before it reads. */
apack_status apack_workspace_size(const apack_seqs *seqs, size_t *bytes);

/* Keep counts of Eq. inner, ceil((1-P)|S|), from keep ratios r = 1-P.
   keep_ratio_h: [B][2] (audio, visual) in [0, 1]; with APACK_SELECT_JOINT
   only [b][0] is used and applies to |S| = n_audio + n_visual.
   The ratio is read on a 1e-6 grid: k = min(n, ceil(round(r*1e6) * n / 1e6))
   in integer arithmetic, so that 0.55 * 100 keeps 55, not 56.
   Outputs (host): keep_count_h [B][2] (JOINT: [b][1] = 0) and
   new_cu_seqlens_h [B+1], the packed offsets after the step. */
apack_status apack_keep_counts(const apack_seqs *seqs, const float *keep_ratio_h, int32_t select_mode,
                               int32_t *keep_count_h, int32_t *new_cu_seqlens_h);

/* Relevance scores of Eq. inner_score (Sec. 3.2), averaged over all Hq query
   heads and all query rows of each sequence:
     I_i = 1/(Hq * n_q) * sum_h sum_r  exp(q_{r,h}.k_{i,g(h)} / sqrt(D))
                                      / sum_{j in S} exp(q_{r,h}.k_{j,g(h)} / sqrt(D))
   for i in S of the sequence, and I_i = 0 for tokens outside S.  With
   seqs->softmax_domain = APACK_SOFTMAX_CAUSAL_ROW the sum in the denominator
   runs over every token j <= p_r (p_r = q_start + r, the row's position within
   its sequence; q_start = len - n_q without seqs->q_start_h) and row r adds to
   I_i only when i <= p_r.
   q: bf16 [sum n_q][Hq][D], contiguous (the query rows at the pruning layer).
   k: bf16 keys of the pruning layer, token t at k + t*k_token_stride, laid
      out [Hkv][D] within the row; k_token_stride a multiple of 16 bytes.
   scores: fp32 [T].  Computed in fp32 from bf16 products on the tensor
   cores; deterministic (fixed reduction order).  q and k must be
   device memory (they are read by TMA; host memory gives APACK_EINVAL). */
apack_status apack_score(const apack_seqs *seqs, const void *q, const void *k, int64_t k_token_stride,
                         float *scores, void *ws, size_t ws_bytes, void *stream);

/* Top-k selection of Eq. inner per segment (see APACK_SELECT_*): keeps the
   keep_count_h[b][m] highest scores of each segment, equal scores going to the
   lower token index, plus every token outside S.
   keep_count_h: host [B][2] counts (JOINT: [b][0] over |S|), or NULL: the
   counts come from keep_ratio_h (host [B][2], the keep ratios 1-P of Eq. inner)
   by the rule of apack_keep_counts.
   Outputs: keep_idx [T_out] (kept token indices in ascending order, i.e. the
   original order; T_out = new_cu_seqlens_h[B] of apack_keep_counts),
   modality_out [T_out] (nullable; the compacted modality mask),
   dst_of_src [T] (nullable; output row of each token or -1),
   new_cu_seqlens [B+1] (nullable; device copy of the new offsets).
   scores must be finite and >= 0 (as apack_score produces). */
apack_status apack_select(const apack_seqs *seqs, const float *scores, const float *keep_ratio_h,
                          const int32_t *keep_count_h, int32_t select_mode, int32_t *keep_idx,
                          uint8_t *modality_out, int32_t *dst_of_src, int32_t *new_cu_seqlens, void *ws,
                          size_t ws_bytes, void *stream);

/* KV-cache and hidden-state slicing (Sec. 3.2, last sentence; Algorithm 1,
   "slice their KV-cache entries"): for every plane of every group,
   dst row j = src row keep_idx[j], j < n_out, bit for bit.
   planes_h: host array of num_groups descriptors.
   In place: a group with src == dst (and equal plane and row strides) is
   compacted within its own buffer.  Output row j reads row keep_idx[j] >= j,
   so each store waits (bounded) until every load that reads the rows it
   overwrites is done; the rows must be 16-byte multiples of at most 32 KB,
   16-byte aligned (APACK_EUNSUPPORTED otherwise), planes must not overlap,
   and ws is required: the launch keeps its progress words or wave counter
   in bytes 256..1023 (the workspace of apack_workspace_size has them).
   Host source: a group whose src is pinned host memory (cudaHostAlloc or
   cudaHostRegister) is gathered over the host link by plain loads (zero
   copy): only the kept rows cross the link.  Its dst must be device memory,
   and it cannot be in place (APACK_EINVAL).
   ws: NULL (out of place only), or a 256-byte aligned workspace (e.g. the
   one of apack_score, at least 1024 bytes) whose error word receives
   APACK_ETIMEOUT if a bounded wait gives up. */
apack_status apack_compact(const int32_t *keep_idx, int64_t n_out, const apack_plane *planes_h,
                           int32_t num_groups, void *ws, void *stream);

/* One pruning step at layer `layer` of a num_layers-layer decoder
   (Algorithm 1, one iteration of the inner-LLM loop): apack_score on the
   layer's keys, apack_select, then compaction of the K and V caches of
   layers [layer, num_layers), of the hidden states and of any extra planes.
   k_cache / v_cache: bf16, slab 0 = layer `layer`, slab i at
     + i*kv_layer_stride bytes, token t at + t*Hkv*D*2 bytes within a slab.
   k_out / v_out: the same layout with kv_out_layer_stride; k_out == k_cache
     and v_out == v_cache with equal strides compact in place (the first T_out
     token rows of every slab, see apack_compact).
   hidden / hidden_out: bf16 [T][hidden_dim] / [T_out][hidden_dim] (hidden may be NULL;
     hidden_out == hidden compacts in place).
   keep_count_h: [B][2] counts (e.g. cumulative schedules); when NULL they
   come from keep_ratio_h as in apack_keep_counts.
   new_cu_seqlens_h (host, [B+1]) receives the new offsets before the call
   returns (no device synchronisation needed).
   scores (device [T] fp32) receives the relevance scores.
   stage_events_h: NULL, or 4 cudaEvent_t recorded on `stream` before
   scoring, before selection, before compaction and at the end.
   Every argument, the compaction groups included, is checked before the
   first launch: a status other than APACK_OK and APACK_ECUDA means nothing
   was queued on `stream`. */
apack_status apack_prune_step(const apack_seqs *seqs, int32_t layer, int32_t num_layers,
                              const void *q, const void *k_cache, const void *v_cache,
                              int64_t kv_layer_stride, const void *hidden, int64_t hidden_dim,
                              const float *keep_ratio_h, const int32_t *keep_count_h, int32_t select_mode,
                              void *k_out, void *v_out, int64_t kv_out_layer_stride, void *hidden_out,
                              const apack_plane *extra_planes_h, int32_t num_extra,
                              uint8_t *modality_out, int32_t *keep_idx, int32_t *new_cu_seqlens_h,
                              int32_t *new_cu_seqlens, float *scores, void *ws, size_t ws_bytes,
                              void *const *stage_events_h, void *stream);

/* apack_score for callers that cannot allocate device memory: plugins inside
   an engine that owns every device allocation, and serving processes that fix
   their device memory at start-up.  The paper has no counterpart; it is a
   deployment variant of apack_score.
   Same arguments, checks and results as apack_score (q and k must be device
   memory: host memory is refused with APACK_EINVAL before any device work),
   without the workspace: the
   scratch is one 8 MiB array that the library keeps on every device it is
   loaded on, until the process exits.  Batches whose apack_workspace_size
   exceeds 8 MiB return APACK_EWORKSPACE (a single 7B-shaped sequence with
   135k tokens and 256 query rows needs about 5.6 MiB).  Nothing is allocated.
   The first call on a device looks the array's address up (a CUDA runtime
   call); make that first call before any stream capture on that device.
   All calls share the one array and it keeps the last call's contents: calls
   that can overlap on the GPU (other streams, other threads) race on it and
   must be serialised by the caller.
   device_error_out: NULL, or a device int32 that receives the call's device
   error code (APACK_OK, APACK_ETIMEOUT, APACK_EDEVICE) on `stream`. */
apack_status apack_score_static(const apack_seqs *seqs, const void *q, const void *k, int64_t k_token_stride,
                                float *scores, int32_t *device_error_out, void *stream);

/* Pre-LLM frame alignment (Sec. 3.1, "Coarse pass" and "Gated fine pass";
   Eq. cka and Eq. gate; Algorithm 1, its first pre-LLM steps).  Per video frame f:
     v_f = mean of the frame's visual tokens; a_f = mean of the audio tokens
           resampled onto the frame axis (audio token j belongs to frame
           floor(j * n_frames / n_audio));
     c_f = ||V_f^T A_f||_F^2 / (||A_f^T A_f||_F ||V_f^T V_f||_F), linear CKA of the
           mean-centred window rows f - window/2 .. f + window/2 (cut to the clip;
           0 for a window whose centred rows vanish);
     s_f = c_f if mean(c) >= tau, else (1 - beta) c_f + beta (1 - dn_f), with
           dn_f = the min-max normalised ||v_f - a_f|| over the clip.
   visual: bf16 [n_frames * tokens_per_frame][dim], frame f's tokens at rows
   f*tokens_per_frame ..; audio: bf16 [n_audio][dim]; dim a multiple of 8,
   n_audio >= n_frames >= 1, window odd in 1..7 (the paper uses 3, tau = 0.78,
   beta = 0.90).  Outputs (device, fp32): c_out [F], s_out [F], dnorm_out [F]
   (nullable), cbar_out [1] (nullable).  fp32 accumulation, fixed reduction
   order (deterministic).  ws: 256-byte aligned, apack_frame_alignment_workspace_size
   bytes, not zeroed: every call writes the device error word in its first 16
   bytes (apack_device_error).  A device-side wait that runs out records
   APACK_ETIMEOUT there, and every output of the call is NaN. */
apack_status apack_frame_alignment_workspace_size(int32_t n_frames, int64_t dim, size_t *bytes);
apack_status apack_frame_alignment(const void *visual, const void *audio, int32_t n_frames,
                                   int32_t tokens_per_frame, int32_t n_audio, int64_t dim, int32_t window,
                                   float tau, float beta, float *c_out, float *s_out, float *dnorm_out,
                                   float *cbar_out, void *ws, size_t ws_bytes, void *stream);

/* ---- A whole progressive schedule in one call.
   Sec. 3.2: pruning is repeated at later layers, each step keeping a fraction of
   the current tokens (Algorithm 1, the inner-LLM loop).  Step i does what
   apack_prune_step does at layer steps_h[i].layer; its inputs are step i-1's
   outputs (K/V from k_out/v_out at layer offset l_i - l_(i-1), hidden_out,
   modality_out, new_cu_seqlens_h, and the counts kept as the new audio/visual
   counts; (|S|, 0) in joint mode).  Layers are strictly ascending.  Each step
   needs its own keep_idx; outputs of step i+1 may reuse step i-1's buffers
   (ping-pong).  All steps (queries and compaction groups included) are
   checked on the host before the first launch;
   then everything runs in order on `stream` (bit-identical to one
   apack_prune_step per step).  stage_events_h: NULL or 4*num_steps events
   (entries may be NULL), recorded for step i before scoring [4i], after
   scoring [4i+1], after selection [4i+2] and after compaction [4i+3].  ws must
   hold apack_workspace_size of every step's sequences. */
typedef struct apack_step {
  int32_t layer;                   /* pruning layer l_i */
  const void *q;                   /* bf16 [sum n_q][Hq][128]: query rows of layer l_i */
  const int32_t *keep_count_h;     /* host [B][2] kept tokens after the step, or NULL */
  const float *keep_ratio_h;       /* host [B][2] keep ratios, used when keep_count_h is NULL */
  void *k_out, *v_out;             /* bf16 [L - l_i][T_i][Hkv][128] */
  int64_t kv_out_layer_stride;     /* bytes between layers of k_out / v_out */
  void *hidden_out;                /* bf16 [T_i][hidden_dim]; required when hidden is given */
  const apack_plane *extra_planes_h; /* further per-token planes of this step, or NULL */
  int32_t num_extra;
  uint8_t *modality_out;           /* [T_i] */
  int32_t *keep_idx;               /* [T_i] */
  int32_t *new_cu_seqlens_h;       /* host [B+1], written by the call */
  int32_t *new_cu_seqlens;         /* device [B+1] or NULL */
} apack_step;

apack_status apack_prune_schedule(const apack_seqs *seqs, int32_t num_layers, const void *k_cache,
                                  const void *v_cache, int64_t kv_layer_stride, const void *hidden,
                                  int64_t hidden_dim, int32_t select_mode, const apack_step *steps_h,
                                  int32_t num_steps, float *scores, void *ws, size_t ws_bytes,
                                  void *const *stage_events_h, void *stream);

/* ---- The schedule as a CUDA graph.
   apack_prune_schedule_graph makes the same checks and host planning as
   apack_prune_schedule (same arguments, no stage events) once, and captures its
   launches into an executable CUDA graph; it launches nothing itself.  It
   writes steps_h[i].new_cu_seqlens_h as the direct call does.
   apack_graph_launch replays those launches on `stream`, with the same
   pointers, sizes and keep counts: one graph launch instead of one launch per
   kernel, for a schedule that repeats with fixed shapes (a serving bucket).
   Every device buffer named at capture must stay allocated while the graph is
   used; the host-side arguments are not read again after the capture returns.
   apack_graph_destroy frees the graph.  Errors: the capture's own checks
   (as apack_prune_schedule), APACK_ECUDA if the driver refuses the capture. */
typedef struct apack_graph_s *apack_graph;
apack_status apack_prune_schedule_graph(const apack_seqs *seqs, int32_t num_layers, const void *k_cache,
                                        const void *v_cache, int64_t kv_layer_stride, const void *hidden,
                                        int64_t hidden_dim, int32_t select_mode, const apack_step *steps_h,
                                        int32_t num_steps, float *scores, void *ws, size_t ws_bytes,
                                        apack_graph *graph_out);
apack_status apack_graph_launch(apack_graph graph, void *stream);
apack_status apack_graph_destroy(apack_graph graph);

/* ---- Decode-step attention over a (compacted) KV cache.
   Sec. 3.2 (last sentence) and App. G: pruning shortens the cache that every
   autoregressive decode step attends to.  One decode token per sequence:
     out[b][h][:] = sum_j softmax_j(q[b][h] . k[j][g] / sqrt(128)) v[j][g][:],
   g = h / (Hq / Hkv), j over all cu_seqlens_h[b] .. cu_seqlens_h[b+1]-1
   (every cached token, not only the multimodal ones).
   q: bf16 [num_seqs][Hq][128] (8-byte aligned); k, v: bf16 token rows
   [T][Hkv][128] with kv_token_stride bytes between tokens (16-byte aligned,
   a multiple of 16, >= Hkv*256); out: fp32 [num_seqs][Hq][128] (16-byte
   aligned, device).  cu_seqlens_h: host [num_seqs+1], starting at 0; an
   empty sequence gives zeros.  Supported: Hq / Hkv <= 8 and Hkv in
   {1, 2, 4, 8} (APACK_EUNSUPPORTED otherwise).  fp32 accumulation.  With
   Hkv 2 or 4 and at most 8 query heads per KV head (the tensor-core path) the
   CTAs of a sequence claim its 128-key tiles from a counter as they go, so
   the grouping of keys into partial sums, and with it the last bits of out,
   can differ from call to call (not where the caches are so short that each
   CTA has its own tiles); the other head layouts merge in a fixed order.
   ws: 256-byte aligned, apack_decode_workspace_size bytes (the size depends
   on the device's SM count: query it on the device that runs the call),
   zeroed by the caller once before its first use: its first 16 bytes are a
   device error word read by apack_device_error, and bytes 256..511 hold the
   claim counters, which every call leaves at zero.  Batch, caches and ws_bytes
   may change from call to call on one workspace; the size for the longest
   caches serves every shorter one of as many sequences.  A device-side wait that
   runs out records APACK_ETIMEOUT there.  Two kernel launches per 64
   sequences; no allocation, no synchronisation. */
apack_status apack_decode_workspace_size(int32_t num_seqs, const int32_t *cu_seqlens_h, int32_t num_q_heads,
                                         int32_t num_kv_heads, size_t *bytes);
apack_status apack_decode_attention(int32_t num_seqs, const int32_t *cu_seqlens_h, const void *q, const void *k,
                                    const void *v, int64_t kv_token_stride, int32_t num_q_heads,
                                    int32_t num_kv_heads, float *out, void *ws, size_t ws_bytes, void *stream);

/* ---- Paged key-value caches.
   Sec. 3.2 drops tokens "together with their key-value entries": what a step frees is of use to other
   sequences only where a cache is kept in pages.  A pool holds num_pages pages of page_tokens tokens for
   every layer; row r of sequence b is slot r % page_tokens of page
   page_table[b*table_stride + r/page_tokens].  Token rows of a page may lie [token][head][D] or
   [head][token][D], pages and layers in either order: the strides say so.  One page that holds a whole
   contiguous cache is a pool too (num_pages 1, page_tokens T), so that contiguous caches and pages are
   sources and destinations of the same calls.

   The device memory that the calls below are given is the current device's.

   Element types of the calls below. */
enum { APACK_BF16 = 0, APACK_FP16 = 1, APACK_FP32 = 2 };

typedef struct apack_paged_cache {
  void *k, *v;                  /* layer 0, page 0, token 0, head 0; device memory, 16-byte aligned */
  int64_t layer_stride;         /* bytes, multiples of 16, the same for k and v; of the last four a stride */
  int64_t page_stride;          /*   whose extent is 1 is not read.  Heads and tokens of a page must not */
  int64_t token_stride;         /*   overlap, nor pages and layers of the pool (APACK_EINVAL) */
  int64_t head_stride;
  int32_t num_layers, num_pages;
  int32_t page_tokens;          /* tokens per page, 1 .. 2^30 */
  int32_t num_kv_heads;         /* 1 .. 256 */
  int32_t head_dim;             /* D: 64 or 128 (APACK_EUNSUPPORTED otherwise) */
  int32_t dtype;                /* APACK_BF16 or APACK_FP16 */
  const int32_t *page_table;    /* device [num_seqs][max_pages]; entries behind a sequence's last row are not read */
  int64_t table_stride;         /* int32 entries between the rows of page_table, >= max_pages */
  int32_t num_seqs;             /* 1 .. APACK_MAX_SEQS */
  int32_t max_pages;            /* columns of page_table, >= 1 */
} apack_paged_cache;

/* Rotary positions.  Pair i of a head's first rotary_dim elements turns by the angle
   t = positions[axis(i)][token] * freq_h[i]:
     (a, b) -> magnitude * (a cos t - b sin t, b cos t + a sin t);
   APACK_ROTARY_HALF pairs elements (i, i + rotary_dim/2), APACK_ROTARY_PAIRS elements (2i, 2i + 1); the
   elements from rotary_dim on pass unchanged.  With num_axes 2 or 3 (time, height and width of a visual
   token) the first section[0] pairs take their position from axis 0, the next section[1] from axis 1 and so
   on; the sections add up to rotary_dim/2.  Angles are reduced modulo one turn in 64-bit fixed point, so
   that far positions keep them to 2^-24 of a turn, whatever int32 the position is and for frequencies of up to
   2^40 radians (twice as far off for each doubling beyond); arithmetic in fp32, one rounding. */
enum { APACK_ROTARY_HALF = 0, APACK_ROTARY_PAIRS = 1 };
typedef struct apack_rotary_spec {
  int32_t layout;               /* APACK_ROTARY_* */
  int32_t rotary_dim;           /* even, 2 .. head_dim */
  int32_t num_axes;             /* 1 .. 3 */
  int32_t section[3];           /* pairs per axis, >= 0; not read when num_axes is 1 */
  float magnitude;              /* finite */
  const double *freq_h;         /* HOST [rotary_dim/2], radians per position, finite; read before the call returns */
} apack_rotary_spec;

/* The frequencies freq_h[i] = base^(-2i/rotary_dim) and their forms for contexts `factor` times longer than
   the original_len tokens that a model was trained on:
     LINEAR  freq / factor (position interpolation);
     NTK     base * factor^(r/(r-2)) in the place of base, r = rotary_dim >= 4;
     YARN    (arXiv 2309.00071, Eqs. 10-13) freq * g + freq / factor * (1 - g), where g rises from 0 to 1
             as the turns original_len * freq / 2 pi of the pair rise from beta_slow to beta_fast;
             magnitude = 0.1 ln(factor) + 1.
   magnitude_h receives 1 in the other forms.  Host only. */
enum { APACK_ROTARY_NONE = 0, APACK_ROTARY_LINEAR = 1, APACK_ROTARY_NTK = 2, APACK_ROTARY_YARN = 3 };
apack_status apack_rotary_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor,
                                      int64_t original_len, double beta_fast, double beta_slow, double *freq_h,
                                      float *magnitude_h);

/* Rotates num_heads heads of D elements in each of n_tokens rows.  x: token t's heads, back to back, at
   x + t*x_token_stride bytes; out likewise; out == x with equal strides rotates in place, and no row of out may
   overlap one of x otherwise (APACK_EINVAL).  positions: int32, axis a's position of token t at
   positions[a*pos_axis_stride + t]; pos_axis_stride >= n_tokens, or 0: one position for all axes (a text token).
   transpose non-zero: the transposed map, the gradient with respect to x of a rotation (it turns back by the
   same angles and keeps the magnitude).  dtype: APACK_BF16, APACK_FP16 or APACK_FP32.  head_dim: 2 .. 256,
   even.  x and out aligned to the element; 16-byte aligned rows and rotary_dim, head_dim multiples of 16 take
   wide loads.  n_tokens up to 2^31 - 1; 0 does nothing. */
apack_status apack_rotary(const apack_rotary_spec *spec, int32_t dtype, int64_t n_tokens, int32_t num_heads,
                          int32_t head_dim, const void *x, int64_t x_token_stride, void *out, int64_t out_token_stride,
                          const int32_t *positions, int64_t pos_axis_stride, int32_t transpose, void *stream);

/* A decode step's or a prompt's new tokens: rotates their queries into q_out and their keys into the pages of
   `layer`, and writes their values there.  Token t goes to row rows[t] of sequence seqs[t] (seqs NULL: of
   sequence t, n_tokens <= num_seqs); a negative row writes neither key nor value (padding of a captured batch;
   its query is rotated all the same).  No two tokens of a call may name one slot.  q [n][num_q_heads][D] (at
   any token stride, as k and v: slices of one projection's output), q_out likewise (q_out == q with equal strides in
   place; otherwise no row of it may overlap one of q, k or v, APACK_EINVAL), k and v [n][num_kv_heads][D]; dtype and D of the cache; every pointer and stride a multiple of 16
   bytes.  spec NULL: nothing is rotated.  num_q_heads 0 .. 1024; with 0, q and q_out are NULL (keys and values
   alone).
   ws: NULL, or a workspace whose error word (its first 16 bytes) receives APACK_EDEVICE when a row lies behind
   the page table or a page number outside the pool; such a token is not written, with or without ws. */
apack_status apack_rotary_append(const apack_rotary_spec *spec, const apack_paged_cache *cache, int32_t layer,
                                 int64_t n_tokens, const void *q, int64_t q_token_stride, void *q_out,
                                 int64_t q_out_token_stride, int32_t num_q_heads, const void *k,
                                 int64_t k_token_stride, const void *v, int64_t v_token_stride,
                                 const int32_t *positions, int64_t pos_axis_stride, const int32_t *rows,
                                 const int32_t *seqs, void *ws, void *stream);

/* apack_decode_attention over pages: one token per sequence,
     out[b][h] = sum_r softmax_r(scale q[b][h] . k[r][g]) v[r][g],  g = h / (Hq / Hkv), r < seqlens[b],
   the lengths on the DEVICE, so that a captured call follows growing caches.  An empty sequence gives zeros
   and an lse of -infinity; what lies behind a sequence's last row (infinities and NaN too) has no influence.
   A NaN or infinity among the rows themselves makes what it enters NaN (an infinite value: infinite or NaN).
   q: [num_seqs][Hq][D] at q_token_stride bytes, cache dtype, 16-byte aligned; scale > 0, finite times log2(e)
   too (1/sqrt(D) is usual).
   out: [num_seqs][Hq][D], contiguous, 16-byte aligned, out_dtype the cache's or APACK_FP32; it must not overlap q
   (APACK_EINVAL).  lse: fp32
   [num_seqs][Hq] or NULL, ln sum_r exp(scale q.k).  Hq / Hkv <= 32 (APACK_EUNSUPPORTED otherwise), Hq <= 1024.
   fp32 softmax and accumulation; the sums' order depends on the lengths alone (deterministic).
   A length below 0 or above max_pages*page_tokens is read as the nearest of the two, and a page number outside
   the pool as a page of zeros; both record APACK_EDEVICE in the error word of ws.  So do lengths (over shared pages)
   whose list of work passes 2^31 - 1025 entries, and the outputs of sequences that are not empty are left as they are.
   With h the largest divisor of Hkv up to 8 (up to 4 if Hq / Hkv > 16), a sequence of n > 0 tokens has
   Hkv / h * (ceil(n D / 2048) + 24 / h) entries (24 / h rounded down), and the first 24 / h are not counted: some 3.4e10
   tokens for D = 128 and Hkv up to 8, 1.4e8 for 251 KV heads.
   ws: 256-byte aligned, apack_paged_decode_workspace_size bytes (for this pool and Hq, whatever the lengths;
   query it on the device that runs the call), its error word (first 16 bytes) zeroed once by the caller.
   Two captured graphs may share a workspace as long as they do not overlap.  Two kernel launches. */
apack_status apack_paged_decode_workspace_size(const apack_paged_cache *cache, int32_t num_q_heads, size_t *bytes);
apack_status apack_paged_decode_attention(const apack_paged_cache *cache, int32_t layer, const int32_t *seqlens,
                                          const void *q, int64_t q_token_stride, int32_t num_q_heads, float scale,
                                          void *out, int32_t out_dtype, float *lse, void *ws, size_t ws_bytes,
                                          void *stream);

/* ---- Attention over shared rows.
   Sequences that were forked from one (questions about one video) hold the same first pages, and one decode token each is
   not all that a step brings: a question's tokens enter together, and so does a part of a long prompt.
   apack_paged_group_plan lays out a step's work from lengths and groups on the DEVICE, once for all layers;
   apack_paged_group_attention runs it on a layer:
     out[t][h] = sum_r softmax_r(scale q[t][h] . k[r][g]) v[r][g],  g = h / (Hq / Hkv),  r <= position of token t,
   for the new tokens t of every sequence of the batch, whose keys and values are in the cache already.

   The batch: n_seqs entries (1 .. APACK_MAX_SEQS); entry e is sequence seqs[e] of the cache (device [n_seqs]; NULL:
   sequence e), with seqlens[seqs[e]] rows (device [num_seqs]; 0 .. min(max_pages * page_tokens, 2^30)).  Its new tokens are
   the last of them: token cu_q[e] + i (device [n_seqs + 1], rising from 0; NULL: one token each, n_q = n_seqs) is row
   seqlens - m + i, of m = cu_q[e+1] - cu_q[e].  q has n_q tokens, cu_q[n_seqs] <= n_q; what lies behind them is neither
   read nor written (padding of a captured batch).  A token that sees no row gives zeros and an lse of -infinity.
   Groups: group i is entries cu_groups[i] .. cu_groups[i+1] - 1 (device [n_groups + 1], rising, 0 .. n_seqs; entries outside
   share nothing; n_groups 0: none).  The caller says with prefix[i] (device [n_groups]) that the first prefix[i] rows of all
   of them are the same: they may be read once for all, through the first entry's row of the page table (its length at least
   prefix[i]).  Whether they are is the plan's choice (not where every sequence has many new tokens of its own), so that
   every entry's row of the table is complete all the same; what is read together changes the result by rounding only.
   An entry or a group that these words do not allow records APACK_EDEVICE in the error word of ws: a length or a prefix out
   of range is read as the nearest in range, tokens before a sequence's first row see nothing, an entry outside the cache
   gives zeros; offsets that do not rise leave no plan, and the attention calls then record APACK_EDEVICE and write nothing.
   So do calls that do not match the plan's n_q, heads, D or cache geometry.

   q: [n_q][Hq][D] at q_token_stride bytes, cache dtype, 16-byte aligned; scale as in apack_paged_decode_attention; out:
   [n_q][Hq][D], contiguous, cache dtype, 16-byte aligned, not over q; lse: fp32 [n_q][Hq] or NULL, ln sum_r exp(scale q.k).
   Hq <= 1024, any Hq / Hkv; n_q * Hq <= 2^28, n_q <= 2^24.  fp32 softmax and accumulation; deterministic.
   A page number outside the pool is read as a page of zeros and recorded.  What a token does not see (rows behind it,
   behind the sequence's last, NaN and infinities too) has no influence on it; a NaN or infinity among the rows that
   it sees makes what it enters NaN (an infinite value: infinite or NaN).
   ws: 256-byte aligned, apack_paged_group_workspace_size bytes (for at most n_seqs entries and n_q tokens; query it on the
   device that runs the calls), its error word (first 16 bytes) zeroed once by the caller.  The plan and the parts of unfinished
   sums live in it: calls of one plan follow each other on one stream, no other call uses the workspace between them, and
   another plan in it ends the first.  One launch for a plan, two for a layer.
   Probabilities enter the product with the values as one 16-bit number each.  A step of one token per sequence that shares
   little (fewer than some 10 sequences on 5,000 rows, 5 on 23,000, or nothing) is faster, and keeps 24 bits of them, in
   apack_paged_decode_attention. */
apack_status apack_paged_group_workspace_size(const apack_paged_cache *cache, int32_t num_q_heads, int32_t n_seqs,
                                              int64_t n_q, size_t *bytes);
apack_status apack_paged_group_plan(const apack_paged_cache *cache, const int32_t *seqlens, int32_t num_q_heads,
                                    int32_t n_seqs, const int32_t *seqs, const int32_t *cu_q, int64_t n_q,
                                    int32_t n_groups, const int32_t *cu_groups, const int32_t *prefix, void *ws,
                                    size_t ws_bytes, void *stream);
apack_status apack_paged_group_attention(const apack_paged_cache *cache, int32_t layer, int64_t n_q, const void *q,
                                         int64_t q_token_stride, int32_t num_q_heads, float scale, void *out, float *lse,
                                         void *ws, size_t ws_bytes, void *stream);

/* apack_compact between pools: row j - cu_dst[b] of dst's sequence b receives, for K and V of num_layers
   layers (src_layer and dst_layer on), bit for bit, row
     keep_idx[j] - cu_src[b]   (keep_idx as apack_select writes it, packed over the batch; cu_src: the packed
                                offsets that entered the step, device [B+1])
     keep_idx[j]               where cu_src is NULL (one page that holds the packed batch)
     j - cu_dst[b]             where keep_idx is NULL (every sequence's first rows; cu_src must be NULL)
   of src's sequence b, for j in [cu_dst[b], cu_dst[b+1]); cu_dst: device [B+1], apack_select's new_cu_seqlens.
   n_out: cu_dst[B], or an upper bound of it (keep_idx is read below cu_dst[B] alone).  B = num_seqs of both
   pools; heads, D and dtype equal; page sizes and strides may differ.  Slots of dst that no j names keep what
   they hold.
   Out of place (another pool, other pages of the same one by another table, or other layers), no page that is
   written may be read by the same call.  In place: src and dst name the same pool, table and layers; keep_idx is
   then given and strictly ascending within each sequence, and each sequence's pages are its own; rows move towards the
   front of their sequence.
   ws: NULL, or a workspace whose error word receives APACK_EDEVICE when a row lies behind a page table or a
   page number outside its pool; such a row is not copied, with or without ws. */
apack_status apack_paged_compact(const apack_paged_cache *src, const apack_paged_cache *dst, int32_t src_layer,
                                 int32_t dst_layer, int32_t num_layers, const int32_t *keep_idx,
                                 const int32_t *cu_src, const int32_t *cu_dst, int64_t n_out, void *ws, void *stream);

/* Copies page pairs[i][0] to page pairs[i][1] in every layer, K and V, i < n_pairs (device int32 [n_pairs][2]):
   the pages that a forked sequence needs of its own.  No page may be written twice, nor written and read by
   the same call; a pair of one page with itself is padding, reads and writes nothing and may stand beside any other.
   page_table is not read and may be NULL.
   ws as in apack_paged_compact; a pair with a page outside the pool is not copied. */
apack_status apack_copy_pages(const apack_paged_cache *cache, const int32_t *pairs, int64_t n_pairs, void *ws,
                              void *stream);

/* ---- Page tables kept on the device.
   Who holds which page: the page tables and lengths of up to num_seqs sequences, how many sequences hold each page
   (refs; 0: a free page), and a stack of the free pages (free_list[0 .. *free_count - 1], the last on top).  The calls
   below change them with kernels, from device arrays, so that a captured step of a server (new tokens, questions that
   come and go) needs neither the host nor fixed lengths.  All are int32 device memory of the caller's, 4-byte aligned;
   page_table and lengths are those that apack_paged_cache and the attention calls read.  Start: lengths 0, refs 0,
   free_list all pages, *free_count num_pages.  One call at a time may change them (calls on one stream).
   In every call: n entries, 0 .. APACK_MAX_SEQS; seqs (device [n]): the sequence of an entry, NULL: entry i is sequence i
   (n <= num_seqs); no sequence twice.  Rows to keep or to add may be entries of lengths, as they are before the call; no
   other list of a call lies in the tables' memory.  An entry that cannot be carried out (a sequence outside the table or
   named twice, rows or pages that it does not have, pages that are wanted and not free, a page of the table that nobody
   holds) leaves everything as it was, and records APACK_EDEVICE in the error word of ws (NULL, or a 16-byte aligned
   workspace) for the whole call.  Which pages a call takes and leaves depends on its arguments and the state alone
   (deterministic).  n = 0 does nothing, except that apack_pages_extend writes its maps. */
typedef struct apack_page_tables {
  int32_t *page_table;          /* [num_seqs][max_pages]; -1 where a sequence has no page */
  int64_t table_stride;         /* int32 entries between its rows, >= max_pages */
  int32_t *lengths;             /* [num_seqs] rows of each sequence; ceil(rows / page_tokens) pages are held */
  int32_t *refs;                /* [num_pages] */
  int32_t *free_list;           /* [num_pages] */
  int32_t *free_count;          /* [1] */
  int32_t num_seqs;             /* 1 .. APACK_MAX_SEQS */
  int32_t max_pages;            /* columns of page_table, >= 1 */
  int32_t num_pages;            /* >= 1 */
  int32_t page_tokens;          /* 1 .. 2^30 */
} apack_page_tables;

/* Every entry keeps its first keep_rows[i] rows (device [n], 0 .. its length; 0: the sequence ends).  The pages behind them
   are given up; those that no other sequence holds become free, the call's first on top of the stack (in the order of
   entries, then of rows), so that an extension by as many pages takes the same ones to the same places. */
apack_status apack_pages_release(const apack_page_tables *tables, int32_t n, const int32_t *seqs, const int32_t *keep_rows,
                                 void *ws, void *stream);

/* Entry i's sequence, which must be empty, shares the pages and takes the length of sequence parents[i] (device [n]; a parent
   may be named often).  seqs is not NULL. */
apack_status apack_pages_fork(const apack_page_tables *tables, int32_t n, const int32_t *parents, const int32_t *seqs,
                              void *ws, void *stream);

/* Room for new_rows[i] >= 0 more rows behind each entry's, in pages from the top of the stack (in the order of entries, then of
   rows).  A partly filled last page that other sequences hold too is not written to: the entry gets a page of its own in its
   place, first of its pages, and pairs[i] = (old, new) for apack_copy_pages, (0, 0) elsewhere, which copies nothing (int32
   [n][2], 8-byte aligned; with NULL an entry that needs a page of its own cannot be carried out).  Of the sequences that
   share it, all that the call extends get their own but the last holder.
   The map of the new rows, packed over the entries: cu_new (int32 [n+1]) their offsets; rows[j] (int32 [max_rows]) the row in
   its sequence, row_seqs[j] (int32 [max_rows] or NULL) that sequence, as apack_rotary_append takes them; slots[j] (int64
   [max_rows], 8-byte aligned, or NULL) page * page_tokens + slot in the page.  Behind the last new row, and all of them in
   a call that cannot be carried out: -1 (padding of a captured batch), cu_new 0 in the latter.  More than max_rows new rows cannot be
   carried out.  One kernel launch, two with max_rows above 8192. */
apack_status apack_pages_extend(const apack_page_tables *tables, int32_t n, const int32_t *seqs, const int32_t *new_rows,
                                int32_t *cu_new, int64_t max_rows, int32_t *rows, int32_t *row_seqs, int64_t *slots,
                                int32_t *pairs, void *ws, void *stream);

/* Synchronises `stream`, then reads the device error word of `ws` into
   *code_out (APACK_OK, APACK_ETIMEOUT or APACK_EDEVICE) and clears it when
   `clear` is non-zero. */
apack_status apack_device_error(const void *ws, void *stream, int32_t *code_out, int32_t clear);

/* Number of kernels this library has launched in the calling process. */
uint64_t apack_launch_count(void);

/* Human-readable name of a status code (static string). */
const char *apack_status_string(apack_status status);

#ifdef __cplusplus
}
#endif

#endif /* APACK_H */
