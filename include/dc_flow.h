/*
 * dc_flow.h — C ABI of the MI355X streaming flow-decoder chunk step.
 *
 * The flow decoder is the stage of the Token2Wav pipeline before the vocoder:
 * it turns the token encoder's features mu (n_mel values per frame) into mel
 * frames by conditional flow matching.  One call integrates dx/dt = v(x, t)
 * from Gaussian noise at t = 0 to t = 1 in n_steps explicit Euler steps on a
 * cosine time grid; v is the classifier-free-guided combination
 * (1 + w) v_cond - w v_uncond of a DiT estimator evaluated on the conditional
 * input (x | mu | speaker | prompt mel) and the unconditional one (x | 0 | 0 |
 * 0) (Motivation, "Where the time goes": a CFM solve with CFG x2 per second
 * of speech; Design, "Adapter": n_steps = 10).  Each attention of each block
 * at each solver step also attends to that step's carry: the keys and values
 * of the turn's prompt and of the last f_retained / f_chunk chunks, which the
 * call itself writes in place (the stacked carry of Design, "State rule",
 * Eq. carry: new frames in front, the immutable prompt tail behind, extent
 * capped at L = f_retained + f_prompt; the attended extents are f_prompt,
 * f_prompt + f_chunk, ..., L, Eq. catalog).  The whole call for f_call frames
 * -- n_steps x (input projection, depth x 5 kernels, output projection,
 * guided Euler update) -- is one HIP graph replay (Design, "Granularity and
 * capture placement", Eq. granularity: binding at the chunk clock divides
 * host launches by n_steps).
 *
 * Shapes fixed by the kernels: head width dim / heads = 64 and dim <= 512;
 * mlp a multiple of 32; n_mel a multiple of 8, <= 1024; t_dim even, <= 1024.
 *
 * Conventions are those of dc.h: functions return a dc_status (0 on
 * success); dc_flow_last_error() explains the last failure; a state is not
 * thread-safe; the state owns one device arena whose addresses are fixed
 * until dc_flow_free.  All tensor arguments are device pointers in
 * row-major float32 unless DC_HOST_PTRS is set in flags (then host pointers,
 * and every call is synchronous).
 */
#ifndef DC_FLOW_H
#define DC_FLOW_H

#include <stddef.h>
#include <stdint.h>

#include "dc.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DC_FLOW_ABI_VERSION 1

typedef struct dc_flow_cfg {
    int32_t abi_version;                 /* DC_FLOW_ABI_VERSION                                   */
    int32_t n_mel, dim, heads, depth;    /* estimator: mel bins, width, heads (dim/heads = 64),   */
    int32_t mlp, t_dim;                  /*   blocks, MLP width, sinusoidal time-embedding width  */
    int32_t n_steps;                     /* Euler solver steps per call                           */
    int32_t f_prompt;                    /* largest prompt, frames                                */
    int32_t f_retained;                  /* history frames kept in the carry (multiple of f_chunk)*/
    int32_t f_chunk;                     /* frames a full call retains (its advance)              */
    int32_t f_call;                      /* largest call: f_chunk plus the lookahead              */
    int32_t batch;                       /* independent streams decoded together                  */
    int32_t dtype;                       /* DC_F32 or DC_BF16 (bf16 operands, fp32 accumulation)  */
    uint32_t flags;                      /* DC_HOST_PTRS, DC_NO_GRAPH                             */
    float cfg_rate;                      /* guidance weight w                                     */
    float temperature;                   /* scale of the initial noise                            */
    uint64_t rng_seed;                   /* first key word of the noise generator                 */
    void* hip_stream;                    /* hipStream_t to run on; NULL = a stream of the state's own */
} dc_flow_cfg;

typedef struct dc_flow_stats {
    int64_t calls;            /* dc_flow_decode_chunk calls that launched work                  */
    int64_t replays;          /* calls served by the captured f_call-frame graph                */
    int64_t direct;           /* calls launched kernel by kernel (other n, or DC_NO_GRAPH)       */
    int64_t prompts;          /* dc_flow_prompt calls                                            */
    int64_t rejected;         /* calls refused by argument checks                               */
    int64_t weight_bytes;     /* device bytes of weights and per-step constants                 */
    int64_t carry_bytes;      /* device bytes of the stacked carry (all streams)                */
    int64_t carry_live_bytes; /* bytes of the carry's declared live extent L (all streams)      */
    int64_t arena_bytes;      /* total device bytes of the state                                */
    int32_t kernels_per_call; /* kernel launches of one f_call-frame call                       */
    int32_t graph_nodes;      /* nodes of the captured graph (0 without one)                    */
    double capture_ms;        /* dc_flow_init wall time: upload, constants, warm-up, capture     */
} dc_flow_stats;

/* Device time of one kernel role in one call (dc_flow_profile). */
typedef struct dc_flow_kernel_stat {
    char name[48];            /* role: "assemble", "gemm:in", "gemm:qkv", "attn", "gemm:o",
                                 "heads" (with options), "gemm:fc1", "gemm:fc2", "gemm:out", "euler"                           */
    int32_t launches;         /* launches of this role per call                                      */
    int32_t mfma;             /* 1: the role is a matrix-core contraction                            */
    double us;                /* device time per call, summed over its launches (HIP events)        */
    double flops;             /* algorithmic floating-point operations per call                      */
    double bytes;             /* algorithmic HBM bytes per call: operands read once, results written */
} dc_flow_kernel_stat;

typedef struct dc_flow_state dc_flow_state;

/* Number of float32 values the weight blob of cfg must hold (0 for NULL).  The
 * blob holds, back to back in PyTorch Linear layouts [out][in]: the time MLP
 * (t.W1 [dim][t_dim], t.b1, t.W2 [dim][dim], t.b2), the input projection
 * (in.W [dim][4 n_mel], in.b), per block (ada.W [6 dim][dim], ada.b,
 * qkv.W [3 dim][dim], qkv.b, o.W [dim][dim], o.b, fc1.W [mlp][dim], fc1.b,
 * fc2.W [dim][mlp], fc2.b) and the final layer (ada.W [2 dim][dim], ada.b,
 * out.W [n_mel][dim], out.b). */
int64_t dc_flow_blob_floats(const dc_flow_cfg* cfg);

/* Create a state: validate cfg, upload the weights (host float32 blob of
 * blob_bytes bytes; rounded to bfloat16 for a DC_BF16 state's per-step Linear
 * layers), compute the per-step time modulations on the device, zero the
 * carry, and capture the f_call-frame call as one graph.  No stream has a
 * turn yet.  Errors: DC_EINVAL (bad cfg or blob size), DC_EVERSION,
 * DC_ENOMEM, DC_EDEVICE. */
dc_status dc_flow_init(const void* weights_blob, size_t blob_bytes, const dc_flow_cfg* cfg, dc_flow_state** out);

/* Options of dc_flow_init_opt.
 *
 * qk_norm: every block normalises its queries and keys per head (RMS norm,
 * eps qk_eps, with a gain per dimension) and rotates the first rope_dims of
 * a head's 64 dimensions by the frame's position since the turn start: pair j
 * is dimensions (j, j + rope_dims / 2), its frequency rope_base^(-2 j /
 * rope_dims) radians a frame, rounded to float32 (dc_qk_norm_rope below).  The
 * blob then holds, behind the tensors of dc_flow_blob_floats, the gains
 * [depth][2][64] (queries, keys).  The carry holds keys as they are attended
 * to, normalised and rotated.
 *
 * carry_bits 4: the stacked carry is held in 4 bits (dc_carry4 below: E2M1
 * with one scale for 32 values): 34 bytes per head, frame and key or value
 * instead of 128 (bf16) or 256.  A call's own frames are stored first and
 * attended to as they are held. */
#define DC_FLOW_OPT_VERSION 1
typedef struct dc_flow_opt {
    int32_t abi_version;      /* DC_FLOW_OPT_VERSION                                         */
    int32_t carry_bits;       /* 0: the carry in the operand type; 4                         */
    int32_t qk_norm;          /* 0 or 1                                                      */
    int32_t rope_dims;        /* 0 (norm only) .. 64, a multiple of 16; 0 without qk_norm    */
    float rope_base;          /* > 0, finite, with rope_dims                                 */
    float qk_eps;             /* >= 0, finite, with qk_norm                                  */
} dc_flow_opt;

/* dc_flow_blob_floats and dc_flow_init with options (NULL: none, the same as
 * without).  Errors as theirs; DC_EVERSION also for opt's. */
int64_t dc_flow_blob_floats_opt(const dc_flow_cfg* cfg, const dc_flow_opt* opt);
dc_status dc_flow_init_opt(const void* weights_blob, size_t blob_bytes, const dc_flow_cfg* cfg, const dc_flow_opt* opt,
                           dc_flow_state** out);

/* Start a turn of stream b: the prompt pass over `frames` frames (1 <=
 * frames <= f_prompt; mu and cond [frames][n_mel], spk [n_mel]) writes the
 * prompt's keys and values of every solver step, block and guidance branch
 * in place as the stream's whole carry (the turn transition of Design,
 * "State rule": base state written into existing storage), and restarts the
 * stream's frame position and history.  Other streams are untouched.  Errors:
 * DC_EINVAL (NULL pointer, b or frames out of range), DC_ESTATE, DC_EDEVICE. */
dc_status dc_flow_prompt(dc_flow_state* s, int32_t b, const float* mu, const float* cond, const float* spk,
                         int32_t frames);

/* One chunk call for every stream: mu [batch][n][n_mel] are the features of
 * frames [p_b, p_b + n) of each stream (p_b = the stream's position), mel_out
 * [batch][n][n_mel] receives the solved mel frames.  1 <= n <= f_call; every
 * stream must have a turn.  When n >= f_chunk the first f_chunk frames of
 * each stream enter its carry and its position advances by f_chunk (the rest
 * are the lookahead, presented again by the next call); a call of fewer
 * frames is a flush that changes no state.  n == f_call replays the captured
 * graph.  Errors: DC_EINVAL, DC_ERANGE (n out of range), DC_ESTATE (a stream
 * without a turn, or a poisoned state), DC_EDEVICE. */
dc_status dc_flow_decode_chunk(dc_flow_state* s, const float* mu, int32_t n, float* mel_out);

/* Wait for the state's stream. */
dc_status dc_flow_sync(dc_flow_state* s);

/* The carry of stream b for (solver step, block, branch 0 = conditional /
 * 1 = unconditional, kv 0 = keys / 1 = values) in Eq. carry's logical order
 * (newest retained chunk first, the prompt last), widened to float32 into the
 * host buffer host_out [frames][dim]; *frames receives the extent.  Pass
 * host_out = NULL to query the extent.  For audits against the definition
 * (the shadow auditor of Design, "Verification"); synchronous.  Errors:
 * DC_EINVAL, DC_EDEVICE. */
dc_status dc_flow_carry_read(dc_flow_state* s, int32_t b, int32_t step, int32_t layer, int32_t branch, int32_t kv,
                             float* host_out, int32_t* frames);

dc_status dc_flow_get_stats(const dc_flow_state* s, dc_flow_stats* out);

/* Time an f_call-frame call launch by launch, `reps` times (mean per call),
 * with HIP events on the state's stream, grouped by kernel role into out[0 ..
 * *count) (at most max entries; out = NULL queries the count).  The streams'
 * state does not advance and no retained frame changes: the call writes only
 * the slot that the next call overwrites.  Every stream needs a turn.  For
 * measurement; synchronous.  Errors: DC_EINVAL, DC_ESTATE, DC_EDEVICE. */
dc_status dc_flow_profile(dc_flow_state* s, int32_t reps, dc_flow_kernel_stat* out, int32_t max, int32_t* count);

/* Text of the last error of s (of the last failed dc_flow_init when s is NULL). */
const char* dc_flow_last_error(const dc_flow_state* s);

/* Release the state and its device memory.  NULL is a no-op. */
void dc_flow_free(dc_flow_state* s);

/* ------------------------------------------------ attention operators
 *
 * What a streaming transformer's attention needs around its Linear layers,
 * over tensors of the caller's: per-head norms with the position rotation, a
 * carry of keys and values held in 4 bits, and the attention over that carry.
 * A flow decoder made by dc_flow_init_opt runs the same kernels.
 *
 * Entries.  A call works on `batch` entries (streams) of `n` tokens each.
 * Token i of entry e stands at position pos[e] + i.  With `lens`, entry e has
 * only its first lens[e] tokens (0 .. n); rows behind them are neither read
 * nor written.  These arrays are read on the device, so a captured call takes
 * their values at each replay.  Values out of range are taken as the nearest
 * that is in range; an entry with a negative position, or one past 2^60, has
 * no tokens.
 *
 * The carry keeps, per entry and key head, the first `sinks` tokens of a turn
 * (the prompt) in slots of their own and the tokens after them in a ring of
 * `ring` slots: position p >= sinks lies in ring slot (p - sinks) mod ring.  An
 * entry may keep fewer first tokens (`sinks` of dc_span); it has to use the
 * same number in every call of the turn.  The memory is the caller's
 * (dc_carry4_bytes), needs no initial value, and holds no position or length:
 * a call reads and writes exactly what its spans say, and a slot that no call
 * has written is read only if a span names its position.
 *
 * Elements are OCP Microscaling E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
 * negatives) with one scale for 32 consecutive dimensions: 2^e, e the least
 * integer in [-126, 126] for which 6 * 2^e is at least the group's largest
 * magnitude; ties to the even code.  4.25 bits a value.  A group with a NaN
 * or an infinity is held as NaN, and one with a magnitude of 3.5 * 2^126 and
 * more, which rounds to 2^128, as well.
 *
 * Every call is launched on hip_stream, a stream of the current device, and
 * returns without waiting; nothing is allocated, so calls can be captured.
 * The device pointers have to be the current device's.  Errors: DC_EINVAL
 * (nothing is launched), DC_ERANGE (a size past the kernels' limits),
 * DC_EDEVICE; dc_carry4_last_error() explains the last one of the calling
 * thread. */

#define DC_CARRY4_ABI_VERSION 1

typedef struct dc_carry4 {
    int32_t abi_version;      /* DC_CARRY4_ABI_VERSION                                          */
    int32_t batch, heads;     /* entries, key / value heads                                     */
    int32_t head_dim;         /* 64 or 128                                                      */
    int32_t sinks, ring;      /* slots of first tokens (>= 0), ring slots (>= 1); sum <= 2^24   */
    void* data;               /* device, dc_carry4_bytes() bytes, 256-byte aligned              */
} dc_carry4;

typedef struct dc_span {
    const int64_t* pos;       /* device [batch]: position of each entry's first token of the call */
    const int32_t* lens;      /* device [batch]: tokens of each entry, or NULL: n each          */
    const int32_t* sinks;     /* device [batch]: first tokens kept, or NULL: the carry's sinks  */
    int32_t batch, n;         /* entries, tokens of a call                                      */
} dc_span;

/* Rows of heads: head h of token i of entry e at data + e stride_b + i
 * stride_t + h stride_h, in elements; a row's head_dim elements are
 * consecutive.  Rows aligned to 16 bytes are read and written in 16-byte
 * words, others element by element. */
typedef struct dc_head_rows {
    void* data;
    int64_t stride_b, stride_t, stride_h;
    int32_t heads;
} dc_head_rows;

/* Per-head RMS norm and rotation: y = x / sqrt(mean(x^2) + eps) * gain; then
 * pair j of the first 2 n_freqs dimensions turns by position * freqs[j]:
 * (a, b) -> (a cos - b sin, b cos + a sin), a = y[j], b = y[j + n_freqs], or
 * y[2 j], y[2 j + 1] interleaved.  Dimensions past 2 n_freqs are only
 * normalised.  The angle is taken in 64 bits. */
typedef struct dc_qk_norm {
    const float* q_gain;      /* device [head_dim], or NULL: ones                               */
    const float* k_gain;
    const float* freqs;       /* device [n_freqs], radians a position                           */
    int32_t n_freqs;          /* a multiple of 8, 2 n_freqs <= head_dim; 0: no rotation         */
    int32_t interleaved;
    float eps;                /* >= 0                                                           */
} dc_qk_norm;

/* q_out, k_out = norm and rotation of q, k (head_dim 64 or 128, dtype DC_F32
 * or DC_BF16; sums in fp32, one rounding).  An output may be its input (the
 * same rows); otherwise rows may not overlap.  A row's mean square plus eps has
 * to be a normal fp32 number: larger rows give 0, smaller ones infinities. */
dc_status dc_qk_norm_rope(const dc_qk_norm* norm, const dc_span* span, int32_t head_dim, int32_t dtype,
                          const dc_head_rows* q, const dc_head_rows* k, const dc_head_rows* q_out,
                          const dc_head_rows* k_out, void* hip_stream);

/* Device bytes of the carry (0 for a carry that the calls refuse; data may be NULL). */
int64_t dc_carry4_bytes(const dc_carry4* c);

/* Store the span's keys and values.  With norm, q and k are normalised and
 * rotated in the same pass: q_out receives the queries, and the keys are
 * stored from their unrounded values; q and q_out are NULL without norm.  A
 * call may hold more tokens than the ring: of tokens that share a slot the
 * last one is stored. */
dc_status dc_carry4_append(const dc_carry4* c, const dc_qk_norm* norm, const dc_span* span, int32_t dtype,
                           const dc_head_rows* q, const dc_head_rows* k, const dc_head_rows* v,
                           const dc_head_rows* q_out, void* hip_stream);

/* out = softmax(scale q k^T) v of the span's queries over the carry, which has
 * to hold the call's own tokens already (dc_carry4_append with the same span).
 * q->heads is a multiple of the carry's heads; query head h reads key head
 * h / (q->heads / heads).  A query at position p sees the first tokens and
 *   causal:  of both those up to p, and of the others the positions > p - window
 *            (window >= 1);
 *   else:    the positions in [pos - window, pos + len) of its entry, the same
 *            for all its queries (window >= 0),
 * as far as the ring still holds them after the call's last token: size it for
 * window + n tokens (causal: one less).  A call that begins among the first
 * tokens needs as many slots less as it stores there, so windows and calls of
 * up to ring + sinks are taken; longer ones are refused (DC_ERANGE).  A query
 * that sees nothing gives 0, one whose scores are infinite NaN.
 * out's rows may be q's.
 * workspace: dc_carry4_workspace() device bytes, 16-byte aligned (NULL where
 * that is 0, as for sizes that the call refuses), not shared with a call that
 * may run at the same time.  Sums and statistics in fp32; with DC_BF16 the
 * probabilities are rounded to bf16 for the product with the values, with
 * DC_F32 they are not.  The order of the sums is fixed by the call's sizes
 * (batch, heads, n, window, the carry's slots) and type: the same call gives
 * the same bits, whatever the other entries hold. */
int64_t dc_carry4_workspace(const dc_carry4* c, int32_t q_heads, int32_t n, int32_t window);
dc_status dc_carry4_attend(const dc_carry4* c, const dc_span* span, int32_t dtype, const dc_head_rows* q,
                           const dc_head_rows* out, int32_t window, int32_t causal, float scale, void* workspace,
                           int64_t workspace_bytes, void* hip_stream);

/* The values that the carry holds for the span's tokens (for audits): k, v in
 * dtype (exact in both). */
dc_status dc_carry4_read(const dc_carry4* c, const dc_span* span, int32_t dtype, const dc_head_rows* k,
                         const dc_head_rows* v, void* hip_stream);

/* Text of the calling thread's last error of these calls. */
const char* dc_carry4_last_error(void);

#ifdef __cplusplus
}
#endif

#endif
