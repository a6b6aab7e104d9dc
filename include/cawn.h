/*
 * libcawn -- causal phase accumulation of the CAWN Resonance Layer on NVIDIA B200 (sm_100a).
 *
 * C ABI.  Every pointer is caller-owned; "device" pointers are CUDA global memory of the
 * current device, "host" pointers are ordinary (preferably pinned) host memory.  The
 * library calls no allocator, and its scratch lives in a caller-provided workspace, with two
 * exceptions that keep state inside the library: cawn_phase_accumulate_fwd_host creates, on its
 * first large call per device, two copy streams and a handful of events that it keeps and
 * serialises behind a lock; cawn_phase_accumulate_fwd_static uses a 4 MiB __device__ array that
 * is part of the library image and shared by all calls on a device (serialise them).
 * Calls are asynchronous on the given CUDA stream
 * (a cudaStream_t passed as void*; NULL = the legacy default stream) unless stated.
 *
 * Shapes.  B batch, L time steps, H heads, F harmonics per head, C = H*F complex channels,
 * flat channel index j = h*F + k.  "complex64" = two consecutive floats (re, im).
 *   pushes / outputs / gradients   [B, L, C] complex64, C contiguous
 *   states                         [B, C]    complex64
 *   gamma, theta                   [C]       float   (retention, rotation in rad/step)
 *   gate mask                      [B, L, ceil(C/32)] uint32, bit (j%32) of word j/32
 * Arrays of shape [B,L,*] and the workspace must be 16-byte aligned, the others 8-byte.
 *
 * The operation (paper: Section "Causal Phase Accumulation and Positional Injection").
 *   z_t   = p_t if |p_t| >= gate_eps else 0               hard-threshold gate
 *   P_t   = z_t + gamma_j e^{i theta_j} P_{t-1}           Eq. (phase_accum_r), Eq. (phase_accum_i)
 *   P_-1  = state_in (0 when NULL)
 *   y_t   = clamp(P_t, +-clamp_abs) component-wise        Eq. (phase_clamp); output only
 *   state_out = P_{L-1}, never clamped                    O(1) state passing
 * All arithmetic is float32 on float32 data; per-channel coefficients are prepared in
 * double inside the kernels.
 *
 * Errors.  Every entry point returns a cawn_status.  Negative values mean the call was
 * rejected before anything was launched.  Conditions found on the device (a carry wait that
 * ran out) are recorded in the workspace and read with cawn_poll_status().  Nothing aborts,
 * traps or waits without a bound.
 */
#ifndef CAWN_H_
#define CAWN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define CAWN_API __attribute__((visibility("default")))
#else
#define CAWN_API
#endif

typedef enum cawn_status {
    CAWN_OK                       = 0,
    CAWN_ERR_INVALID_ARG          = -1,  /* bad struct_size, negative size, unknown op/flag     */
    CAWN_ERR_NULL_POINTER         = -2,  /* a required pointer is NULL                           */
    CAWN_ERR_MISALIGNED           = -3,  /* a pointer breaks the alignment rule above            */
    CAWN_ERR_UNSUPPORTED          = -4,  /* valid request this build has no kernel for           */
    CAWN_ERR_WORKSPACE_TOO_SMALL  = -5,
    CAWN_ERR_CUDA                 = -6,  /* a CUDA runtime call failed (launch, copy)            */
    CAWN_ERR_STATIC_TOO_LARGE     = -7,  /* cawn_phase_accumulate_fwd_static: the call needs more
                                            scratch than the library's built-in array holds      */
    CAWN_ERR_CARRY_TIMEOUT        = 1,   /* device: an inter-tile carry wait hit its bound;
                                            outputs of that call are incomplete                  */
    CAWN_STATUS_NONFINITE         = 2    /* device: an Inf or NaN was accumulated (an Inf input, a
                                            non-finite carried state, an overflow); outputs are
                                            complete but contain such values.  NaN pushes alone do
                                            not raise it: they fail the gate's comparison and are
                                            dropped.  The two device conditions are bits: a poll may
                                            return 3 when both occurred.                          */
} cawn_status;

enum {
    CAWN_FLAG_PRELUDE_CLAMP_SILU = 1u << 0, /* fused path: clamp conv output to +-50, then SiLU   */
    CAWN_FLAG_RETENTION_DYNAMIC  = 1u << 1, /* gamma_t = sigmoid(gamma_logit[b,t,h] + freq_bias[k]) */
    CAWN_FLAG_INPUT_INDEPENDENT  = 1u << 2, /* forward: the caller vouches that `input`, gamma, theta
                                               (and the conv weights) are not written by the call
                                               made just before this one on the same stream, nor, where
                                               that one has this flag too, by the call before it, and so
                                               on back to and including the last call without it (any
                                               of the library's calls; other work in between ends the
                                               chain).  The
                                               kernels are launched so that a call may start while the
                                               previous one drains (programmatic dependent launch);
                                               with this flag the new call also fetches its input rows
                                               during that overlap.  States, masks, workspaces and all
                                               outputs are only touched once the previous call is
                                               complete, with or without the flag.                    */
    CAWN_FLAG_INPUT_BF16         = 1u << 3, /* forward: `input` is stored as bfloat16 (Cartesian: pairs
                                               (re, im) of bf16, 4 bytes per channel; fused path: one
                                               bf16 per channel) and widened, exactly, to float on load */
    CAWN_FLAG_OUTPUT_BF16        = 1u << 4  /* forward: `y` is stored as pairs (re, im) of bfloat16,
                                               each component rounded to nearest even from the fp32
                                               result.  With either flag the recurrence, the carried
                                               state, state_out and the conv history stay fp32 (the
                                               paper runs a bf16 network around an fp32 scan:
                                               Section "Mixed-Precision and Float32
                                               Stabilization").  With the time-varying retention or the
                                               Ear epilogue (the paper's own layer form) the two flags
                                               come together or not at all; the Ear's z_conv is then
                                               bfloat16 [B, L, 2, H, K].  Not available for the
                                               host-staged forward or any backward:
                                               CAWN_ERR_UNSUPPORTED.                                    */
};

/* Operation selector of cawn_workspace_bytes(). */
enum {
    CAWN_OP_FWD        = 0,  /* workspace of cawn_phase_accumulate_fwd                           */
    CAWN_OP_BWD_SAVED  = 1,  /* workspace of cawn_phase_accumulate_bwd with CAWN_SAVED_STATES    */
    CAWN_OP_BWD_PUSHES = 2,  /* ... with CAWN_SAVED_PUSHES (adds room for the recomputed states) */
    CAWN_OP_STATE      = 3,  /* size of one state blob                                           */
    CAWN_OP_FWD_HOST   = 4,  /* device staging + workspace of cawn_phase_accumulate_fwd_host     */
    CAWN_OP_MIXING_BWD = 5   /* workspace of cawn_mixing_bwd                                     */
};

/* What the backward was given to rebuild P_{t-1} from. */
enum {
    CAWN_SAVED_STATES = 0,   /* the forward's unclamped outputs P [B,L,C]                        */
    CAWN_SAVED_PUSHES = 1    /* the forward's input pushes p [B,L,C]; P is recomputed            */
};

/* Plain-data description of one call.  Fill struct_size with sizeof(cawn_params). */
typedef struct cawn_params {
    uint32_t struct_size;
    int32_t  B;              /* batch >= 1                                                       */
    int64_t  L;              /* time steps of this call, >= 0, any value (ragged is fine)        */
    int32_t  H, F;           /* C = H*F >= 1                                                     */
    float    gate_eps;       /* hard-gate threshold on |p| (fused path: on the magnitude m);
                                0 = always open                                                  */
    float    gate_tau;       /* fused path only: logit(gate_eps) rounded to float by the caller;
                                the gate is decided as conv_output >= gate_tau                   */
    float    clamp_abs;      /* output clamp bound (paper: 100); <= 0 disables                   */
    float    grad_clamp_abs; /* backward: clamp returned grad_p and grad_gamma (paper: 100);
                                <= 0 disables                                                    */
    int32_t  conv_k;         /* fused path: conv taps 1..4; 0 = input is Cartesian pushes        */
    uint32_t flags;          /* CAWN_FLAG_*                                                      */
} cawn_params;

/* State blob: P [B,C] complex64 (unclamped), then, at the next 16-byte boundary, the conv
 * history [B, conv_k-1, C] float (raw hidden rows; absent when conv_k <= 1).  This is the
 * fixed-size state the paper carries between chunks, micro-batches and decode steps
 * (Section "Theoretical Advantages", O(1) state passing; Section "Throughput and
 * Autoregressive Efficiency", the 2-step conv history).                                        */

CAWN_API const char *cawn_status_string(int status);

/* Host-only size query.  *bytes receives the size for `op` at these params. */
CAWN_API int cawn_workspace_bytes(const cawn_params *params, int op, size_t *bytes);

/* Zero a freshly allocated workspace (device).  Must run once before its first use; afterwards
 * the kernels keep it consistent themselves.  One workspace serves one call at a time: calls
 * that may overlap on the device need a workspace each.                                         */
CAWN_API int cawn_workspace_init(void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Forward phase accumulation (Eq. (gated_push_r/i) gate, Eq. (phase_accum_r/i), Eq. (phase_clamp)).
 *
 * conv_k == 0:  `input` = pushes p [B,L,C] complex64 (device).  y may alias input.
 * conv_k >= 1:  fused Resonance mixing path.  `input` = hidden states h [B,L,C] float (device);
 *               u_t = bias + sum_k conv_w[c,k] h[t-(conv_k-1)+k]   (causal depthwise conv,
 *               Section "Temporal Syntax Cache"; rows left of t=0 from the state blob or zero),
 *               optional clamp+-50 and SiLU, magnitude m = sigmoid(x), phase = pi*tanh(x),
 *               gate, z = m (cos, sin)(phase).
 * gamma/theta:  [C] device.  With CAWN_FLAG_RETENTION_DYNAMIC gamma is ignored and
 *               gamma_logit [B,L,H], freq_bias [F] (device) define the retention
 *               (Section "Multi-Head Dynamic Parameter Projection", item 4); available for
 *               both input forms (with conv_k >= 1 this is the paper's own layer: Temporal
 *               Syntax Cache, gated push and per-token retention in one pass).
 * state_in:     state blob (device) or NULL for a zero state.
 * y:            [B,L,C] complex64 (device), clamped if clamp_abs > 0.
 * state_out:    state blob (device) or NULL.  May alias state_in.
 * gate_mask:    bit-packed mask (device) or NULL.
 * workspace:    device, >= cawn_workspace_bytes(CAWN_OP_FWD), initialised once.
 */
CAWN_API int cawn_phase_accumulate_fwd(const cawn_params *params,
                                       const void *input,
                                       const float *gamma, const float *theta,
                                       const float *conv_w, const float *conv_bias,
                                       const float *gamma_logit, const float *freq_bias,
                                       const void *state_in,
                                       void *y, void *state_out, uint32_t *gate_mask,
                                       void *workspace, size_t workspace_bytes,
                                       void *cuda_stream);

/*
 * Backward of the Cartesian forward (the reverse-time adjoint the paper's custom autograd
 * function computes, Section "Complex Domain Synthesis and Hardware Compilation").
 *   lam_t = grad_y_t + conj(a) lam_{t+1},  lam_{L-1} = grad_y_{L-1} + grad_state_out
 *   grad_p_t = lam_t at every position (straight-through gate; clamp passes gradient)
 *   grad_gamma_j = sum_{b,t} Re(conj(lam_t) e^{i theta_j} P_{t-1})
 *   grad_theta_j = sum_{b,t} Re(conj(lam_t) i a_j P_{t-1})
 *   grad_state_in = conj(a) lam_0
 * saved / saved_kind: CAWN_SAVED_STATES -> the forward's UNCLAMPED y; CAWN_SAVED_PUSHES -> the
 *               forward's pushes (re-gated and re-scanned into the workspace first).
 * grad_y:       [B,L,C] complex64 (device).  grad_p may alias it.
 * grad_state_out, state_in: [B,C] complex64 (device) or NULL (= 0).
 * grad_gamma, grad_theta: [C] float (device) or NULL.  grad_state_in: [B,C] complex64 or NULL.
 * Deterministic: partial sums are combined in a fixed order in double.
 * Static retention only (see cawn_phase_accumulate_bwd_dynamic for the other form).
 */
CAWN_API int cawn_phase_accumulate_bwd(const cawn_params *params,
                                       const void *saved, int saved_kind,
                                       const float *gamma, const float *theta,
                                       const void *state_in,
                                       const void *grad_y, const void *grad_state_out,
                                       void *grad_p, float *grad_gamma, float *grad_theta,
                                       void *grad_state_in,
                                       void *workspace, size_t workspace_bytes,
                                       void *cuda_stream);

/*
 * Backward with the paper's time-varying retention (Section "Multi-Head Dynamic Parameter
 * Projection", item 4: gamma_{t,h,k} = sigmoid(W_gamma x_t + b_k), the projection per head and a
 * static per-harmonic bias).  params->flags must carry CAWN_FLAG_RETENTION_DYNAMIC.
 *   a_t = gamma_t e^{i theta},  lam_t = grad_y_t + conj(a_{t+1}) lam_{t+1}
 *   d gamma_t(b,t,j) = Re(conj(lam_t) e^{i theta_j} P_{t-1}),  s = gamma_t (1 - gamma_t) d gamma_t
 *   grad_gamma_logit[b,t,h] = sum_k s      grad_freq_bias[k] = sum_{b,t,h} s
 *   grad_theta_j = sum_{b,t} Re(conj(lam_t) i a_t P_{t-1})      grad_state_in = conj(a_0) lam_0
 * gamma_logit [B,L,H], freq_bias [F] (device).  grad_gamma_logit [B,L,H] float, grad_freq_bias [F]
 * float, grad_theta [C] float: device or NULL.  Other arguments as cawn_phase_accumulate_bwd.
 * grad_gamma_logit: where a 64-channel group holds whole heads (F divides 64, or C <= 64) every entry
 * is the sum of one warp and is stored; otherwise the call zeroes the array and accumulates with
 * atomic adds, and when a head spans three or more groups (F > 128) its last bits may differ from
 * run to run.  Everything else is bitwise repeatable.
 */
CAWN_API int cawn_phase_accumulate_bwd_dynamic(const cawn_params *params,
                                               const void *saved, int saved_kind,
                                               const float *gamma_logit, const float *freq_bias,
                                               const float *theta, const void *state_in,
                                               const void *grad_y, const void *grad_state_out,
                                               void *grad_p, float *grad_gamma_logit,
                                               float *grad_freq_bias, float *grad_theta,
                                               void *grad_state_in,
                                               void *workspace, size_t workspace_bytes,
                                               void *cuda_stream);

/*
 * Backward of the fused Resonance mixing path (cawn_phase_accumulate_fwd with conv_k >= 1,
 * static retention): the reverse scan with the prelude's chain rule as its epilogue, one pass
 * over grad_y, the saved states and h.
 *   lam   = reverse scan of grad_y (as cawn_phase_accumulate_bwd); it is the gradient of the pushes
 *   magnitude m = sigmoid(x), phase ph = pi tanh(x), push z = m_used (cos ph, sin ph):
 *     d m  = Re(conj(lam) e^{i ph})                    straight-through: flows open or closed
 *     d ph = m_used (-lam_r sin ph + lam_i cos ph)     m_used = m if the gate is open else 0
 *   (the paper's hard-threshold gate with straight-through estimator, Section "Multi-Head Dynamic
 *   Parameter Projection"), through the optional clamp + SiLU and the causal depthwise conv
 *   (Section "Temporal Syntax Cache") to h, conv_w, conv_bias and the carried conv history.
 * h [B,L,C] float, conv_w [C,conv_k], conv_bias [C] or NULL, gamma/theta [C]: as in the forward.
 * saved_states: the forward's UNCLAMPED y [B,L,C] complex64; may be NULL when neither grad_gamma
 *               nor grad_theta is wanted.
 * state_in:     the forward's state blob (its conv history is read) or NULL.
 * grad_y [B,L,C] complex64; grad_state_out: gradient of the forward's state_out blob (state part
 *               and conv-history part, e.g. the next chunk's grad_state_in) or NULL.
 * grad_h [B,L,C] float; grad_conv_w [C,conv_k], grad_conv_bias [C], grad_gamma [C], grad_theta [C]
 *               float or NULL; grad_state_in: state blob of gradients or NULL.  All device.
 * workspace:    >= cawn_workspace_bytes(CAWN_OP_MIXING_BWD), initialised once (carry records, per-tile
 *               partial sums, and the few rows exchanged at tile seams; O(B*C*L/64)).
 * Deterministic (parameter sums: per-CTA partials combined in a fixed order in double).
 */
CAWN_API int cawn_mixing_bwd(const cawn_params *params,
                             const float *h, const float *conv_w, const float *conv_bias,
                             const float *gamma, const float *theta,
                             const void *saved_states, const void *state_in,
                             const void *grad_y, const void *grad_state_out,
                             float *grad_h, float *grad_conv_w, float *grad_conv_bias,
                             float *grad_gamma, float *grad_theta, void *grad_state_in,
                             void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * cawn_mixing_bwd with the paper's time-varying retention (the fused path run with
 * CAWN_FLAG_RETENTION_DYNAMIC, which params->flags must carry): the backward of the whole
 * Resonance mixing step as the paper defines it — Temporal Syntax Cache, gated push, per-token
 * per-head retention (Section "Multi-Head Dynamic Parameter Projection").  gamma_logit [B,L,H],
 * freq_bias [F] replace gamma; grad_gamma_logit [B,L,H] (as in cawn_phase_accumulate_bwd_dynamic)
 * and grad_freq_bias [F] replace grad_gamma; each may be NULL.  Everything
 * else as cawn_mixing_bwd, including the workspace size.
 */
CAWN_API int cawn_mixing_bwd_dynamic(const cawn_params *params,
                                     const float *h, const float *conv_w, const float *conv_bias,
                                     const float *gamma_logit, const float *freq_bias, const float *theta,
                                     const void *saved_states, const void *state_in,
                                     const void *grad_y, const void *grad_state_out,
                                     float *grad_h, float *grad_conv_w, float *grad_conv_bias,
                                     float *grad_gamma_logit, float *grad_freq_bias, float *grad_theta,
                                     void *grad_state_in,
                                     void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Forward with the front of the Convolutional SwiGLU Ear as the scan's epilogue (Eq. (wave_synth)
 * and Section "Projection to Hidden State: The Convolutional SwiGLU Ear", the depth-wise 1-D
 * convolution across the K harmonics).  Everything up to the clamped state y_t is
 * cawn_phase_accumulate_fwd (Cartesian or fused input, static or time-varying retention: with
 * conv_k >= 1 and CAWN_FLAG_RETENTION_DYNAMIC one kernel takes the hidden states through the
 * paper's whole Resonance mixing step up to the Ear's convolution); instead of storing y the
 * kernel writes
 *   Z_t = Concat(Re y_t, Im y_t)  viewed as 2H channels (real heads, then imaginary heads) x K
 *   z_conv[b,t,q,k] = ear_bias[q] + sum_j ear_w[q,j] Z_t[q, k + j - (ear_k-1)/2],  zero outside 0..K-1
 * The paper states neither the tap count nor the padding: taken as ear_k taps (1 or 3; other
 * values -> CAWN_ERR_UNSUPPORTED) with zero padding on both sides, cross-correlation order as in a
 * Conv1d layer.  ear_k = 1 with ear_w = 1 and no bias gives the planar Z itself.
 * ear_w:   [2H, ear_k] float (device).  ear_bias: [2H] float (device) or NULL.
 * z_conv:  [B, L, 2, H, K] float (device, 16-byte aligned), K = params->F; as many bytes as y.
 *          With CAWN_FLAG_INPUT_BF16 | CAWN_FLAG_OUTPUT_BF16 it holds bfloat16 instead (pass the pointer
 *          as it is).
 * state_out (if given) still receives the unclamped, unconvolved P_{L-1} (and the conv history).
 * Limits: K must divide 64 unless H*K <= 64 (a CTA owns 64 adjacent channels and does not read
 * its neighbours' harmonics).
 * Other arguments, ownership, stream order and status reporting as cawn_phase_accumulate_fwd.
 */
CAWN_API int cawn_phase_accumulate_fwd_ear(const cawn_params *params,
                                           const void *input,
                                           const float *gamma, const float *theta,
                                           const float *conv_w, const float *conv_bias,
                                           const float *gamma_logit, const float *freq_bias,
                                           const void *state_in,
                                           const float *ear_w, const float *ear_bias, int ear_k,
                                           float *z_conv, void *state_out, uint32_t *gate_mask,
                                           void *workspace, size_t workspace_bytes,
                                           void *cuda_stream);

/*
 * Associative combine of two segment summaries (static retention):
 *   state_out = a^n_steps * state_prev + state_local,   a_j = gamma_j e^{i theta_j}
 * where state_local is the end state of an n_steps-long segment run from a ZERO state.  This is
 * the O(1) state passing of the paper composed outside a call (prefill that skips outputs,
 * time sharding).  All states [B,C] complex64 (device); state_out may alias either input.
 * a^n is evaluated in double (pow, sincos), not by repeated multiplication.
 */
CAWN_API int cawn_state_carry(const cawn_params *params,
                              const void *state_prev, const void *state_local,
                              int64_t n_steps,
                              const float *gamma, const float *theta,
                              void *state_out, void *cuda_stream);

/* Synchronise `cuda_stream` and return the device-side status recorded in the workspace by
 * the calls so far (CAWN_OK, or the positive conditions CAWN_ERR_CARRY_TIMEOUT and
 * CAWN_STATUS_NONFINITE or-ed together); the record is then cleared.  This is the hook for the
 * paper's stability protocol (Section "Training Stability in the Complex Domain": skip the step
 * on NaN/Inf), without a pass over the outputs.                                                    */
CAWN_API int cawn_poll_status(void *workspace, void *cuda_stream);

/* Test hook for the bounded waits (no counterpart in the paper).  After this call, in every
 * kernel that uses `workspace`, tile number `withhold_tile` (0-based along time, in the kernel's
 * own tile size: 128 steps in the forward, 64 in the backward, 16 for calls of at most 32 steps)
 * of every (batch, channel group) keeps its summary to itself, and every carry wait gives up
 * after `poll_bound` polls (1..65535; 0 keeps the normal bound).  Tiles that depend on the silent
 * one then run into the bound, record CAWN_ERR_CARRY_TIMEOUT, skip their outputs and pass the
 * failure on; the kernel ends, nothing hangs or traps, and the workspace stays usable.
 * withhold_tile < 0 and poll_bound = 0 switch the hook off.  Stream-ordered.                   */
CAWN_API int cawn_workspace_set_wait_hook(void *workspace, int withhold_tile, unsigned poll_bound,
                                          void *cuda_stream);

/*
 * Host-buffer convenience for the Cartesian forward: copies pushes, gamma, theta (and
 * state_in) from HOST memory to the device staging area, runs the forward, copies y
 * (and state_out, gate_mask) back to HOST memory, all on `cuda_stream`, and returns without
 * synchronising.  `device_scratch` (device, >= cawn_workspace_bytes(CAWN_OP_FWD_HOST), zeroed
 * once with cawn_workspace_init) holds staging and workspace.  Static retention, conv_k == 0.
 * Calls of 8 MB and more are cut into up to 8 slices (batch rows, or for B = 1 stretches of time
 * with the state carried: the paper's chunked prefill) that go through two library-owned copy
 * streams, so that slice i is copied out while slice i+1 is copied in; both streams wait for
 * what precedes the call on `cuda_stream` and `cuda_stream` waits for both before anything
 * after it.  The host buffers should be page-locked for the copies to overlap.  The copy streams
 * and their events are created on the first such call per device (the only resources the
 * library ever creates) and calls that use them are serialised by a lock.
 */
CAWN_API int cawn_phase_accumulate_fwd_host(const cawn_params *params,
                                            const void *p_host,
                                            const float *gamma_host, const float *theta_host,
                                            const void *state_in_host,
                                            void *y_host, void *state_out_host,
                                            uint32_t *gate_mask_host,
                                            void *device_scratch, size_t device_scratch_bytes,
                                            void *cuda_stream);

/*
 * Forward phase accumulation for callers that cannot allocate device memory.  (The paper has
 * no counterpart: this is a packaging variant of cawn_phase_accumulate_fwd, same arithmetic.)
 *
 * Who needs it: code that runs where a cudaMalloc is not an option -- a plugin inside a serving
 * process whose device memory has all been handed to one framework-owned pool, a callback that
 * must not block on the allocator or synchronise the device, or a component that is given
 * input and output buffers and nothing else.  Such a caller cannot provide the carry workspace
 * the ordinary entry point asks for, so this one uses a scratch array compiled into the library
 * instead: a file-scope __device__ array of CAWN_STATIC_SCRATCH_BYTES (4 MiB), which every GPU
 * that loads the library holds until the process exits.
 *
 * Same operation and arguments as the Cartesian, static-retention cawn_phase_accumulate_fwd
 * (conv_k == 0, no CAWN_FLAG_RETENTION_DYNAMIC), without the workspace pair.
 * Anything else (conv_k != 0, CAWN_FLAG_RETENTION_DYNAMIC) is refused with CAWN_ERR_UNSUPPORTED;
 * all arguments are validated before anything is put on the stream.
 * device_status: device pointer to one uint32 or NULL.  When given, the device-side status of
 *               this call is copied there on the stream after the kernel: 0, or the bits
 *               CAWN_ERR_CARRY_TIMEOUT (1) and CAWN_STATUS_NONFINITE (2) or-ed together, as
 *               cawn_poll_status would return them; there is no separate poll call for the
 *               built-in scratch.
 *
 * Limits and rules.
 *  - The call is rejected with CAWN_ERR_STATIC_TOO_LARGE, before anything is launched, when
 *    cawn_workspace_bytes(params, CAWN_OP_FWD) exceeds CAWN_STATIC_SCRATCH_BYTES.  The need is
 *    256 + B * ceil(C/64) * (K + K/7 + 1) * 1024 bytes with K = ceil(L/128) tiles: 1.9 MB for
 *    B=8, L=2048, C=768; about 4,000 (batch x 64-channel group x tile) units in all.
 *  - It calls no cudaMalloc/cudaFree and no allocating library routine.
 *  - The first call on each device looks up the array's device address (one
 *    cudaGetSymbolAddress with that device current) and remembers it; make that first call
 *    outside any stream capture.
 *  - All calls on a device share the one array, and it keeps what the last call left in it.
 *    The kernel's epoch tags make stale records harmless and the status word is cleared at the
 *    start of every call, but two calls that overlap on the GPU (different streams, or
 *    different host threads) race on it: serialise them.
 */
#define CAWN_STATIC_SCRATCH_BYTES (4u << 20)
CAWN_API int cawn_phase_accumulate_fwd_static(const cawn_params *params,
                                              const void *input,
                                              const float *gamma, const float *theta,
                                              const void *state_in,
                                              void *y, void *state_out, uint32_t *gate_mask,
                                              uint32_t *device_status,
                                              void *cuda_stream);

/* ------------------------------------------------------------------------------------------
 * Operators that stand next to the phase accumulation in a layer.  (Not in the paper, which
 * names dropout on the layer's output only.)  The library's rules hold: caller-owned device
 * memory, asynchronous on the given stream, everything validated before anything is launched,
 * 64-bit offsets throughout.  Sequence arrays are float, or bfloat16 with CAWN_FLAG_INPUT_BF16 |
 * CAWN_FLAG_OUTPUT_BF16 (these come together or not at all; other flags are refused); every
 * sum, statistic, state and parameter is float.  All array pointers must be 16-byte aligned.
 * None of these calls keeps anything between calls: a workspace needs no initialisation, and
 * one workspace serves one call at a time.  Results are bitwise repeatable (no atomics).
 * ------------------------------------------------------------------------------------------ */

/*
 * Gated delta rule: per value head a matrix state that decays, and that a new key corrects
 * towards its value instead of adding to it.
 *   S_t = e^{g_t} S_{t-1} + u_t k_t^T
 *   u_t = beta_t (v_t - e^{g_t} S_{t-1} k_t)          S_{-1} = state_in (0 when NULL)
 *   o_t = scale S_t q_t                               state_out = S_{L-1}
 * Shapes.  q, k [B, L, Hk, Dk]; v, o [B, L, Hv, Dv]; g, beta [B, L, Hv] float, dense; states
 * [B, Hv, Dv, Dk] float, dense.  Value head h reads key head h / (Hv/Hk).  The rows of one time step
 * (all heads) are contiguous; consecutive steps lie *_stride elements apart (0 = dense) and batches
 * L times that, so that q, k, v may be slices of one projection's output.
 * g is the log decay, at most 0: e^{g} in [0, 1]; -infinity forgets the state (a packed document's
 * first token).  beta is usually in [0, 1]; the recurrence is stable while beta |k|^2 < 2, which the
 * caller sees to (unit keys).
 * Precision.  Sums are float.  Calls by token (see cawn_delta_rule_step) compute in float throughout.  Calls by chunk
 * multiply on the tensor cores: inputs exactly, computed factors (states, corrections, scores) with 16 or more mantissa
 * bits in bfloat16 storage and 24 in float storage; results are rounded once.  So an error is a part of the terms of a sum,
 * not of a result in which they cancel: of |S| |q| for o, about 2^-17 (float storage 2^-21).  States and the
 * gradients of g and beta come out within 1e-6 to 9e-6 of their norm (float storage: all results, 1e-6 to 4e-6).  The
 * gradient of g is a sum of terms that all carry e^g, so a head with strong decays has it to the same relative accuracy.
 * Non-finite inputs stay in their batch row and value head (v: in their row of the state); a call by chunk may also spoil
 * the tokens before a non-finite one in its chunk of 64, counted from the call's first token.
 * Limits: Hv a multiple of Hk, Dk and Dv multiples of 8 up to 128, strides multiples of 8 elements,
 * B * Hv <= 65535 * 64.
 */
typedef struct cawn_delta_params {
    uint32_t struct_size;
    int32_t  B;              /* batch >= 1                                                       */
    int64_t  L;              /* time steps of this call, >= 0, any value                         */
    int32_t  Hk, Hv;         /* key / query heads, value heads                                   */
    int32_t  Dk, Dv;         /* widths of a key / query and of a value                           */
    float    scale;          /* of the read-out, usually Dk^-1/2                                 */
    uint32_t flags;          /* 0, or CAWN_FLAG_INPUT_BF16 | CAWN_FLAG_OUTPUT_BF16: q, k, v, o and
                                their gradients are bfloat16                                     */
    int64_t  q_stride, k_stride, v_stride, o_stride;   /* elements from one time step to the next; 0 = dense */
} cawn_delta_params;

enum { CAWN_DELTA_FWD = 0, CAWN_DELTA_BWD = 1 };    /* `op` of cawn_delta_rule_workspace_bytes */

/* Host-only size query for cawn_delta_rule_fwd / _bwd; enough for every B and L up to the given ones. */
CAWN_API int cawn_delta_rule_workspace_bytes(const cawn_delta_params *params, int op, size_t *bytes);

/*
 * Forward for prompts and training.  state_in NULL = zero; state_out NULL = not wanted, may alias
 * state_in.  o may not alias an input.  Short calls run the recurrence token by token, longer ones
 * chunk by chunk, and with few heads the time axis is cut into segments that run side by side.
 */
CAWN_API int cawn_delta_rule_fwd(const cawn_delta_params *params,
                                 const void *q, const void *k, const void *v,
                                 const float *g, const float *beta, const float *state_in,
                                 void *o, float *state_out,
                                 void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * The same operation token by token in float32, for decoding: one token (or a few, e.g. a draft
 * that is checked) with the state read and written once.  No workspace.  Any L; meant for short ones.
 */
CAWN_API int cawn_delta_rule_step(const cawn_delta_params *params,
                                  const void *q, const void *k, const void *v,
                                  const float *g, const float *beta, const float *state_in,
                                  void *o, float *state_out, void *cuda_stream);

/*
 * Backward.  Everything is recomputed from the forward's inputs (nothing is saved by the forward).
 * grad_o [B, L, Hv, Dv] (o_stride).  grad_state_out: gradient of state_out or NULL (= 0).
 * grad_q, grad_k [B, L, Hk, Dk] (summed over the value heads that share them), grad_v [B, L, Hv, Dv]:
 * dense, the type of the inputs.  grad_g, grad_beta [B, L, Hv] float.  grad_state_in: float or NULL.
 * Outputs may not alias inputs or each other.
 */
CAWN_API int cawn_delta_rule_bwd(const cawn_delta_params *params,
                                 const void *q, const void *k, const void *v,
                                 const float *g, const float *beta, const float *state_in,
                                 const void *grad_o, const float *grad_state_out,
                                 void *grad_q, void *grad_k, void *grad_v,
                                 float *grad_g, float *grad_beta, float *grad_state_in,
                                 void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Group norm with an activation, channels last: x [N, G*M], statistics over the M channels of each
 * position's group (never over positions, so a causal layer stays causal).
 *   xh = (x - mean) / sqrt(var + eps)      CAWN_NORM_RMS: xh = x / sqrt(mean(x^2) + eps)
 *   z  = xh * weight + bias                [G*M] float each, NULL = 1 and 0
 *   y  = z | z sigmoid(z) | z * gate * sigmoid(gate)          by `act`
 * Heads of a mixer are groups; the rms form with weight = M^-1/2 makes unit queries and keys.
 * x, gate: rows x_stride / gate_stride elements apart (0 = dense).  y and gradients: dense.
 * y may alias x or gate when that one is dense.
 */
enum { CAWN_NORM_ACT_NONE = 0, CAWN_NORM_ACT_SILU = 1, CAWN_NORM_ACT_GATE = 2 };

typedef struct cawn_norm_params {
    uint32_t struct_size;
    int32_t  G;              /* groups >= 1                                                      */
    int64_t  N;              /* positions >= 0                                                   */
    int32_t  M;              /* channels of a group, 1..4096                                     */
    int32_t  act;            /* CAWN_NORM_ACT_*                                                  */
    float    eps;            /* >= 0                                                             */
    int32_t  rms;            /* 0: mean and variance, 1: mean square only                        */
    uint32_t flags;          /* 0, or CAWN_FLAG_INPUT_BF16 | CAWN_FLAG_OUTPUT_BF16               */
    uint32_t reserved;       /* 0                                                                */
    int64_t  x_stride, gate_stride;
} cawn_norm_params;

CAWN_API int cawn_group_norm_fwd(const cawn_norm_params *params, const void *x,
                                 const float *weight, const float *bias, const void *gate,
                                 void *y, void *cuda_stream);

/* Host-only size query for cawn_group_norm_bwd; enough for every N up to the given one. */
CAWN_API int cawn_group_norm_workspace_bytes(const cawn_norm_params *params, size_t *bytes);

/* Backward: grad_y [N, G*M] dense -> grad_x; grad_gate (required with CAWN_NORM_ACT_GATE, NULL
 * otherwise), grad_weight, grad_bias [G*M] float or NULL.  The statistics are recomputed from x.
 * grad_x may alias grad_y.  The workspace is used for grad_weight and grad_bias only and may be NULL
 * when neither is wanted. */
CAWN_API int cawn_group_norm_bwd(const cawn_norm_params *params, const void *x,
                                 const float *weight, const float *bias, const void *gate,
                                 const void *grad_y, void *grad_x, void *grad_gate,
                                 float *grad_weight, float *grad_bias,
                                 void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Dropout whose mask is never stored, with the sum that usually follows:
 *   y_i = residual_i + (keep_i ? x_i / P(keep) : 0)       residual NULL = 0
 * keep_i: 16 random bits of element i are at least T = round(p * 65536).  The bits are those of
 * Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011)
 * with key `seed` and counter (i / 8, offset): word (i % 8) / 2, its low half for even i.  P(keep) =
 * 1 - T / 65536 exactly, so the expectation of y is exact for every p.  The gradient with respect to
 * x is the same call on grad_y with the same seed and offset and no residual.
 * offset_device: device pointer to one uint64 that is added to `offset`, or NULL: a CUDA graph that
 * is replayed gets a new mask by writing it.  y may alias x or residual.
 */
typedef struct cawn_dropout_params {
    uint32_t struct_size;
    float    p;              /* in [0, 1); T is at most 65535                                    */
    int64_t  n;              /* elements >= 0                                                    */
    uint64_t seed, offset;
    uint32_t flags;          /* 0, or CAWN_FLAG_INPUT_BF16 | CAWN_FLAG_OUTPUT_BF16               */
    uint32_t reserved;       /* 0                                                                */
} cawn_dropout_params;

CAWN_API int cawn_dropout(const cawn_dropout_params *params, const void *x, const void *residual,
                          void *y, const uint64_t *offset_device, void *cuda_stream);

/* ------------------------------------------------------------------------------------------
 * Operators of a selective state space layer: a short causal convolution, the scan behind it, and
 * the norm in front of both.  The rules above hold (storage flags, float sums and states, 16-byte
 * aligned pointers unless said otherwise, plain workspaces, no atomics: bitwise repeatable).
 *
 * Sequences.  Arrays of rows hold B sequences, either of L rows each (offsets NULL, rows 0), or
 * packed: `offsets` (device, int64, B + 1 values that do not fall) says that sequence b has the rows
 * offsets[b] .. offsets[b+1] - 1, `rows` how many rows the arrays have, and L how many tokens the
 * longest sequence has.  A sequence may be empty.  The device clamps offsets to the arrays' rows and
 * a sequence to its first L tokens.  Rows that no sequence has are neither read nor written, in no
 * direction.  States have one entry per sequence; an empty sequence passes its state on.
 * ------------------------------------------------------------------------------------------ */

/*
 * Short causal convolution of each channel over time, with its history:
 *   z_t = bias_c + sum_k weight[c,k] x_{t-(K-1)+k}       bias NULL = 0
 *   y_t = z_t | z_t sigmoid(z_t)                         by `act`
 * Rows in front of a sequence are its history state_in [B, K-1, C] float (NULL = 0; the oldest row
 * first); state_out receives the last K-1 rows of (history, sequence) and may alias state_in.
 * x: [rows, C], rows x_stride elements apart (0 = dense), aligned to its elements (whole words are read where
 * rows begin on four of them); y [rows, C] dense, not aliasing x.
 * weight [C, K], bias [C] float.  Single tokens are calls with L = 1.
 */
enum { CAWN_CONV_ACT_NONE = 0, CAWN_CONV_ACT_SILU = 1 };

typedef struct cawn_conv_params {
    uint32_t struct_size;
    int32_t  B;              /* sequences >= 1                                                   */
    int64_t  L;              /* tokens of the longest sequence, >= 0                             */
    int32_t  C;              /* channels >= 1                                                    */
    int32_t  K;              /* taps, 1..4                                                       */
    int32_t  act;            /* CAWN_CONV_ACT_*                                                  */
    uint32_t flags;          /* 0, or CAWN_FLAG_INPUT_BF16 | CAWN_FLAG_OUTPUT_BF16: x, y and their
                                gradients are bfloat16                                           */
    uint32_t reserved[2];    /* 0                                                                */
    int64_t  x_stride;       /* elements from one row of x to the next; 0 = dense                */
    int64_t  rows;           /* packed: rows of the arrays; otherwise 0                          */
} cawn_conv_params;

CAWN_API int cawn_short_conv_fwd(const cawn_conv_params *params, const void *x, const float *weight,
                                 const float *bias, const float *state_in, const int64_t *offsets,
                                 void *y, float *state_out, void *cuda_stream);

/* Host-only size query for cawn_short_conv_bwd; enough for every B and L up to the given ones. */
CAWN_API int cawn_short_conv_workspace_bytes(const cawn_conv_params *params, size_t *bytes);

/* Backward; what the activation needs is recomputed from x.  grad_y, grad_x [rows, C] dense.
 * grad_state_out: gradient of state_out or NULL (= 0).  grad_weight, grad_bias, grad_state_in: float
 * or NULL.  The workspace is used for grad_weight and grad_bias only and may be NULL when neither is
 * wanted.  Outputs may not alias inputs or each other. */
CAWN_API int cawn_short_conv_bwd(const cawn_conv_params *params, const void *x, const float *weight,
                                 const float *bias, const float *state_in, const int64_t *offsets,
                                 const void *grad_y, const float *grad_state_out,
                                 void *grad_x, float *grad_weight, float *grad_bias, float *grad_state_in,
                                 void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Selective scan: per channel c a state of N floats whose decay and input depend on the token.
 *   d_t  = softplus(dt_t + dt_bias), or dt_t + dt_bias with softplus = 0      (dt_bias NULL = 0)
 *   h_t  = exp(d_t A[c,n]) h_{t-1} + d_t x_t B_t[n]                           h_{-1} = state_in (0 when NULL)
 *   y_t  = (sum_n C_t[n] h_t[n] + skip_c x_t) silu(z_t)                       skip NULL = 0; z NULL: no gate
 *   state_out = h_{L-1}
 * Shapes.  x, dt, z, y [rows, D]; B, C [rows, G, N], channel c reads group c / (D/G); A [D, N] float
 * (usually negative; with -infinity a state forgets all, but a step of 0 leaves it as it is); skip, dt_bias [D]
 * float; states [B, D, N] float.  Rows of x, dt, z, B and C lie *_stride elements apart (0 = dense), so that they
 * may be slices of projections, and need only be aligned to their elements (whole words are read where rows begin
 * on 16 bytes; of B and C, on four elements).
 * Precision.  Everything is computed in float; results are rounded once to their type.
 * Where the time axis is cut (see the forward), the product of the decays of a segment's tokens is a float of its own:
 * states that grow (A > 0, or negative steps) by more than 3e38 within one become infinite or NaN, whatever they hold.
 * Non-finite values stay in their sequence and in the channels of their group; gradients of B and C may
 * also be spoilt in the eight tokens, counted from the sequence's first, around one.
 * Limits: N <= 64, G <= 65535.
 */
typedef struct cawn_scan_params {
    uint32_t struct_size;
    int32_t  B;              /* sequences >= 1                                                   */
    int64_t  L;              /* tokens of the longest sequence, >= 0                             */
    int32_t  D;              /* channels >= 1                                                    */
    int32_t  N;              /* states of a channel, 1..64                                       */
    int32_t  G;              /* groups that share B and C; divides D                             */
    int32_t  softplus;       /* 0 or 1                                                           */
    uint32_t flags;          /* 0, or CAWN_FLAG_INPUT_BF16 | CAWN_FLAG_OUTPUT_BF16: x, dt, z, B, C,
                                y and their gradients are bfloat16                               */
    uint32_t reserved;       /* 0                                                                */
    int64_t  x_stride, dt_stride, z_stride, b_stride, c_stride;
    int64_t  rows;           /* packed: rows of the arrays; otherwise 0                          */
} cawn_scan_params;

/* `op` of cawn_selective_scan_workspace_bytes. */
enum {
    CAWN_SCAN_FWD = 0,           /* workspace of cawn_selective_scan_fwd (may be 0 bytes)         */
    CAWN_SCAN_BWD = 1,           /* workspace of cawn_selective_scan_bwd with checkpoints          */
    CAWN_SCAN_BWD_RECOMPUTE = 2, /* ... without: adds room for states that are found again         */
    CAWN_SCAN_CHECKPOINTS = 3    /* size of the checkpoints that a forward can leave for it        */
};

/* Host-only size query; enough for every B, L and rows up to the given ones, packed where they are packed
 * and dense where they are dense. */
CAWN_API int cawn_selective_scan_workspace_bytes(const cawn_scan_params *params, int op, size_t *bytes);

/*
 * Forward for prompts and training.  With few channels and long sequences the time axis is cut into
 * segments that run side by side.  state_in NULL = zero; state_out NULL = not wanted, may alias
 * state_in.  y may not alias an input.  checkpoints: the states of every 16th token, for the backward
 * of the same params and inputs, or NULL.
 */
CAWN_API int cawn_selective_scan_fwd(const cawn_scan_params *params, const void *x, const void *dt, const float *A,
                                     const void *B, const void *C, const float *skip, const float *dt_bias,
                                     const void *z, const float *state_in, const int64_t *offsets,
                                     void *y, float *state_out, float *checkpoints,
                                     void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * The same operation token by token, for decoding: one token (or a few) of B sequences of L tokens each, with
 * the states read and written once.  No workspace.  Any L; meant for short ones.
 */
CAWN_API int cawn_selective_scan_step(const cawn_scan_params *params, const void *x, const void *dt, const float *A,
                                      const void *B, const void *C, const float *skip, const float *dt_bias,
                                      const void *z, const float *state_in,
                                      void *y, float *state_out, void *cuda_stream);

/*
 * Backward.  checkpoints: what the forward left, or NULL (the states are then found again, for the time of
 * about a forward and with the larger workspace).  grad_y [rows, D] dense; grad_state_out: gradient of
 * state_out or NULL (= 0).  grad_x, grad_dt, grad_z [rows, D] and grad_B, grad_C [rows, G, N] (summed over
 * the group's channels): dense, the type of the inputs; grad_z goes with z.  grad_A [D, N], grad_skip,
 * grad_dt_bias [D], grad_state_in [B, D, N]: float; the last three may be NULL.  Outputs may not alias
 * inputs or each other.
 */
CAWN_API int cawn_selective_scan_bwd(const cawn_scan_params *params, const void *x, const void *dt, const float *A,
                                     const void *B, const void *C, const float *skip, const float *dt_bias,
                                     const void *z, const float *state_in, const int64_t *offsets,
                                     const float *checkpoints, const void *grad_y, const float *grad_state_out,
                                     void *grad_x, void *grad_dt, float *grad_A, void *grad_B, void *grad_C,
                                     float *grad_skip, float *grad_dt_bias, void *grad_z, float *grad_state_in,
                                     void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Root-mean-square norm of the stream that a branch is added to:
 *   s = x + residual (residual NULL = 0), rounded to the stream's type;  sum_out = s (NULL = not wanted)
 *   y = s / sqrt(mean(s^2) + eps) * weight                               weight [M] float, NULL = 1
 * x [N, M], rows x_stride elements apart (0 = dense), aligned to its elements; residual, sum_out: [N, M] dense in the stream's
 * type, which is that of x, or float with stream_float.  sum_out may alias residual, or x where x is
 * dense and of the stream's type.  y [N, M] dense, by `out`:
 *   CAWN_NORM_OUT_SAME   the type of x (may alias x where x is dense; scales NULL)
 *   CAWN_NORM_OUT_E4M3   8-bit floats (4 bits of exponent, 3 of mantissa, largest value 448) with a
 *                        scale per scale_block channels of a row (32, 64 or 128; the last may be fewer)
 *                        or per row (0):  scale = max(max |y|, 1e-30) / 448,  stored = y / scale,
 *                        rounded to nearest even from the float value.  scales [N, ceil(M/scale_block)]
 *                        or [N] float.  A NaN in a block makes the block's scale NaN.
 */
enum { CAWN_NORM_OUT_SAME = 0, CAWN_NORM_OUT_E4M3 = 1 };

typedef struct cawn_residual_norm_params {
    uint32_t struct_size;
    int32_t  M;              /* channels, 1..8192                                                */
    int64_t  N;              /* rows >= 0                                                        */
    float    eps;            /* >= 0                                                             */
    int32_t  out;            /* CAWN_NORM_OUT_*                                                  */
    int32_t  scale_block;    /* 0, 32, 64 or 128                                                 */
    int32_t  stream_float;   /* 1: the stream is float though flags say bfloat16                 */
    uint32_t flags;          /* 0, or CAWN_FLAG_INPUT_BF16 | CAWN_FLAG_OUTPUT_BF16               */
    uint32_t reserved;       /* 0                                                                */
    int64_t  x_stride;
} cawn_residual_norm_params;

CAWN_API int cawn_residual_norm_fwd(const cawn_residual_norm_params *params, const void *x, const void *residual,
                                    const float *weight, void *sum_out, void *y, float *scales, void *cuda_stream);

/* Host-only size query for cawn_residual_norm_bwd; enough for every N up to the given one. */
CAWN_API int cawn_residual_norm_workspace_bytes(const cawn_residual_norm_params *params, size_t *bytes);

/* Backward, from the sum that the forward left (`out`, scale_block and x_stride are not looked at: a rounding to 8 bits
 * is passed straight through).  grad_y [N, M] in the type of x; grad_sum: gradient of sum_out in the stream's type,
 * or NULL (= 0).  The gradient of x and of the residual is the same: grad_residual in the stream's type, grad_x in
 * that of x, either may be NULL.  grad_residual may alias grad_sum (and grad_y where the types are the same),
 * grad_x may alias grad_y.  grad_weight [M] float or NULL; the workspace is used for it only. */
CAWN_API int cawn_residual_norm_bwd(const cawn_residual_norm_params *params, const void *sum, const float *weight,
                                    const void *grad_y, const void *grad_sum, void *grad_residual, void *grad_x,
                                    float *grad_weight, void *workspace, size_t workspace_bytes, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* CAWN_H_ */
