/*
 * bimamba.h -- C ABI of the MI355X (gfx950) bidirectional Mamba mixer path.
 *
 * What the library computes (paper Sec. 3.2, eqs. 4-6, and the block variant of Sec. 4.3), per
 * batch element b, direction s in {f (left-to-right), b (right-to-left)}, channel d
 * (head h = d / (d_inner/n_heads), B/C group g = h / (n_heads/n_groups)):
 *
 *   xc_s[t,d] = SiLU(conv_b_s[d] + sum_k conv_w_s[d,k] * x_s[t -/+ (K-1-k), d])      short depthwise conv; causal for f,
 *                                                                                  anti-causal for b; zero outside [0,L)
 *   Delta[t,h] = dt_s[t,h]                       (dt_softplus = 0)
 *              = softplus(dt_s[t,h] + dt_bias_s[h])                (dt_softplus = 1)
 *   h_t[n]    = exp(Delta[t,h] * A_s[h,n]) * h_prev[n] + Delta[t,h] * B_s[t,g,n] * xc_s[t,d]     eq. 4 (t = 0..L-1) / eq. 5 (t = L-1..0)
 *   y_s[t,d]  = sum_n C_s[t,g,n] * h_t[n] + D_s[d] * xc_s[t,d]
 *   g_s[t,d]  = y_s[t,d] * SiLU(z_s[t,d])
 *   out[t,d]  = g_f[t,d] + g_b[t,d]                                                 (BIMAMBA_COMBINE_ADD)
 *   out[t,:]  = [g_f[t,:] | g_b[t,:]]                                               (BIMAMBA_COMBINE_SEPARATE, width 2*d_inner)
 *
 * Eq. 6 adds the two layers' outputs, i.e. after each direction's own output projection.  COMBINE_ADD is that sum only
 * when both directions share one output projection; with untied projections (the paper's setting) use COMBINE_SEPARATE
 * and multiply [g_f | g_b] by the two projection matrices stacked, which realises eq. 6 exactly.
 *
 * With conv_bc = 1 (the Mamba-2 form) B and C pass through the same conv + SiLU as x, using rows
 * d_inner .. d_inner+2*n_groups*d_state-1 of conv_w / conv_b (channel order x | B | C).
 *
 * Memory: every pointer is device memory owned by the caller unless marked "host".  The library allocates nothing and
 * keeps no pointer after a call returns.  What it does keep, per process: per-device caches of launch geometry (the
 * device's CU count, and per kernel variant its occupancy and static LDS), filled the first time a variant is launched
 * on a device, when the library also queries that kernel's attributes and raises its dynamic-LDS limit; the one-shot
 * event pair of bimamba_profile_next_call (per host thread); and the fixed scratch buffer of
 * bimamba_block_fwd_static.  The first-use queries enqueue nothing and are safe under stream capture (a test captures
 * a variant's very first launch).  Activations are token-major with the channel dimension contiguous; batch and token
 * strides are given in elements.
 *
 * Arithmetic: state, decay factors, gate and the sum of eq. 6 are fp32; bf16 I/O is widened on load and rounded
 * to nearest-even once at the final store.  Two kernel families implement the same formulas:
 *   - lane-per-chain kernels (every descriptor): one (direction, batch, channel) recurrence per lane group, all
 *     products and sums in fp32.  When a head's A[h, 0..N-1] is an arithmetic progression in n (checked on the
 *     device, bf16 I/O, d_state <= 32) the N decay factors of a token are formed as a_0 * r^n by repeated
 *     multiplication from two exponentials instead of N exponentials (up to 64 tokens and 16 states: none by
 *     multiplication up to 16384 chains and 0.75 M channel tokens, below 61440 chains at most seven in a row).  (bimamba_bwd, whose results are partly fp32
 *     whatever the I/O dtype, evaluates every exponential.)
 *   - chunked matrix-core kernels (a_kind = SCALAR_PER_HEAD, bf16 I/O, d_state 64 or 128, 32 or 64 channels per
 *     head, time_chunks = state_split = 0): the recurrence over 64-token chunks as dense products on the MFMA
 *     units; their operands (conv output, B, C, the decayed score tile, a copy of the state) are rounded to bf16,
 *     accumulation and the carried state stay fp32.  They read x two channels at a time and the carried state four
 *     states at a time: setting time_chunks or state_split, or passing an x whose pointer is not 4-byte aligned or
 *     whose strides are odd, or an h_in / h_out that is not 16-byte aligned, selects the lane-per-chain kernels for
 *     the call; the workspace size covers both.  A call with few (batch, head) pairs cuts the sequence into time
 *     parts that run concurrently (see bimamba_time_chunks), unless x has a token stride beyond 2^24 elements.
 *
 * Execution: calls validate their arguments on the host, enqueue kernels on the caller's HIP stream
 * and return without synchronising.  Calls on different streams are independent as long as their
 * workspaces do not overlap.
 *
 * Errors: every entry point returns BIMAMBA_OK (0) or a negative bimamba_status.  All codes except
 * BIMAMBA_ERR_HIP are decided on the host before anything is launched.  Nothing throws or aborts.
 */
#ifndef BIMAMBA_H
#define BIMAMBA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define BIMAMBA_VERSION 1

enum bimamba_status {
    BIMAMBA_OK = 0,
    BIMAMBA_ERR_NULL_POINTER = -1,        /* a required pointer is NULL */
    BIMAMBA_ERR_BAD_SHAPE = -2,           /* non-positive or inconsistent dimension, stride smaller than the row */
    BIMAMBA_ERR_UNSUPPORTED = -3,         /* dtype / d_state / d_conv / grouping / token stride / size outside the compiled set */
    BIMAMBA_ERR_MISALIGNED = -4,          /* pointer not aligned to its element size (or 16 bytes for the workspace) */
    BIMAMBA_ERR_WORKSPACE_TOO_SMALL = -5, /* workspace_bytes < bimamba_workspace_bytes() */
    BIMAMBA_ERR_HIP = -6,                 /* a launch of this call failed (errors pending from earlier, unrelated calls are
                                             neither reported nor cleared) */
    BIMAMBA_ERR_SCRATCH_EXCEEDED = -7,    /* bimamba_block_fwd_static: the call needs more than BIMAMBA_STATIC_SCRATCH_BYTES */
    BIMAMBA_ERR_ALIAS = -8                /* what is written may overlap what is read; bimamba_bwd: dpf == dpb (checked on the host) */
};

enum bimamba_dtype { BIMAMBA_F32 = 0, BIMAMBA_BF16 = 1 };
enum bimamba_a_kind {
    BIMAMBA_A_PER_HEAD_STATE = 0,  /* A[n_heads, d_state]; the selective-scan layout has n_heads = d_inner */
    BIMAMBA_A_SCALAR_PER_HEAD = 1  /* A[n_heads]: one decay rate per head (the Mamba-2 form) */
};
enum bimamba_d_kind { BIMAMBA_D_PER_CHANNEL = 0, BIMAMBA_D_PER_HEAD = 1 };
enum bimamba_combine { BIMAMBA_COMBINE_ADD = 0, BIMAMBA_COMBINE_SEPARATE = 1 };

/* Host struct.  Supported: d_state in {4, 8, 16, 32, 64, 128}; 1 <= d_conv <= 4; d_inner % n_heads == 0;
 * n_heads % n_groups == 0; with n_groups > 1, d_inner / n_groups must be a multiple of 64. */
typedef struct bimamba_desc {
    uint32_t struct_size;   /* sizeof(bimamba_desc), checked */
    int32_t batch;          /* >= 0 (0 is a no-op) */
    int32_t seqlen;         /* L >= 0; for bimamba_block_fwd the block length */
    int32_t d_inner;
    int32_t d_state;        /* N */
    int32_t n_heads;        /* H; dt has H channels */
    int32_t n_groups;       /* G; B and C have G*N channels */
    int32_t d_conv;         /* K */
    int32_t io_dtype;       /* bimamba_dtype of x, z, dt, B, C, out, tail_in, tail_out */
    int32_t a_kind;         /* bimamba_a_kind */
    int32_t d_kind;         /* bimamba_d_kind */
    int32_t dt_softplus;    /* 0 or 1 */
    int32_t conv_bc;        /* 0 or 1 */
    int32_t combine;        /* bimamba_combine */
    int32_t time_chunks;    /* 0 = let the library choose; n >= 1 forces the lane-per-chain kernels with n time segments
                               per sequence (segments are scanned in parallel and stitched by a carry pass) */
    int32_t state_split;    /* 0 = let the library choose; 1, 2 or 4 forces the lane-per-chain kernels with that many lanes
                               per (direction, channel) chain, each holding d_state / state_split states (2 needs
                               d_state 16 or 32, 4 needs d_state >= 16); results differ only by the summation order of
                               C_t . h_t */
} bimamba_desc;

/* Per-direction parameters, device pointers, fp32, contiguous.
 * conv_w [conv_ch, d_conv] with conv_ch = d_inner (+ 2*n_groups*d_state if conv_bc); tap d_conv-1 multiplies the
 * current token.  conv_b [conv_ch] or NULL (= 0).  A [n_heads, d_state] or [n_heads].  D [d_inner] or [n_heads].
 * dt_bias [n_heads] or NULL (= 0), read only when dt_softplus = 1. */
typedef struct bimamba_params {
    const float* conv_w;
    const float* conv_b;
    const float* A;
    const float* D;
    const float* dt_bias;
} bimamba_params;

/* One activation tensor [batch, L, channels]: element (b, t, c) lives at ptr + b*stride_batch + t*stride_token + c
 * (in elements of io_dtype).  channels <= stride_token <= 2^26 (BIMAMBA_ERR_UNSUPPORTED beyond: the kernels form row
 * offsets inside a tile of tokens in 32 bits).  Strided views let x, z, dt, B, C be column slices of one projection
 * output.  ptr may be NULL only when batch == 0 or seqlen == 0 (nothing is accessed). */
typedef struct bimamba_tensor {
    void* ptr;
    int64_t stride_batch;
    int64_t stride_token;
} bimamba_tensor;

/* The activations one direction reads: x, z [batch, L, d_inner]; dt [batch, L, n_heads]; B, C [batch, L, n_groups*d_state]. */
typedef struct bimamba_inputs {
    bimamba_tensor x, z, dt, B, C;
} bimamba_inputs;

/*
 * Full-sequence bidirectional mixer path (eqs. 4-6).
 *   desc        host.  pf, pb: host structs of device pointers; pb may equal pf (tied weights).
 *   in_f, in_b  host structs; in_b == NULL or in_b == in_f means both directions read the same activations.
 *   out         [batch, L, d_inner] (ADD) or [batch, L, 2*d_inner] (SEPARATE), io_dtype.  It must not overlap any input
 *               view (BIMAMBA_ERR_ALIAS): byte ranges apart, or, inside one buffer, the same strides (batch stride a
 *               multiple of the token stride) and column ranges apart modulo the token stride.
 *   workspace   device scratch of at least bimamba_workspace_bytes(desc, 0) bytes, 16-byte aligned (may be NULL if 0).
 *   hip_stream  a hipStream_t (NULL = the default stream).
 */
int bimamba_fwd(const bimamba_desc* desc, const bimamba_params* pf, const bimamba_params* pb,
                const bimamba_inputs* in_f, const bimamba_inputs* in_b, const bimamba_tensor* out,
                void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Block variant (Sec. 4.3: the forward state is carried across blocks, right-to-left updates stay inside the
 * block).  desc->seqlen is the block length.  The forward scan starts from h_in and its causal conv sees tail_in
 * to the left of the block; the reverse scan starts from zero at the block's right edge with zeros beyond it.
 *   h_in      fp32 [batch, d_inner, d_state] or NULL (= zero state).
 *   tail_in   io_dtype [batch, d_conv-1, tail_ch], the raw (pre-conv) tokens preceding the block, oldest first, or
 *             NULL (= zeros); tail_ch = d_inner (+ 2*n_groups*d_state if conv_bc, channel order x | B | C).
 *   h_out     fp32 [batch, d_inner, d_state]: forward state after the block's last token, or NULL = do not commit.
 *             May alias h_in.
 *   tail_out  io_dtype, same shape as tail_in: last d_conv-1 raw tokens of (tail_in || block), or NULL.  May alias tail_in.
 * A denoising loop calls this once per step with h_out = tail_out = NULL and commits on the block's last step.
 * Everything else as bimamba_fwd; workspace size is bimamba_workspace_bytes(desc, 1).
 */
int bimamba_block_fwd(const bimamba_desc* desc, const bimamba_params* pf, const bimamba_params* pb,
                      const bimamba_inputs* in_f, const bimamba_inputs* in_b,
                      const float* h_in, const void* tail_in, float* h_out, void* tail_out,
                      const bimamba_tensor* out, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * bimamba_block_fwd for callers that cannot allocate device memory or pass a workspace: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and bit-identical results, but
 * the scratch is a fixed buffer of BIMAMBA_STATIC_SCRATCH_BYTES inside the library's device image (one copy per GPU,
 * held until the process ends); the call allocates and frees nothing.  A descriptor whose
 * bimamba_workspace_bytes(desc, 1) exceeds that size is rejected with BIMAMBA_ERR_SCRATCH_EXCEEDED before anything
 * is launched (batch 16, d_inner 4096 fits blocks of up to 128 tokens in either layout).  All calls on one GPU share
 * the buffer, whatever their stream: two such calls that may overlap in time on the same GPU race; order them on one
 * stream or with events.  Nothing in the buffer has to survive from one call to the next, and nothing in it has to be
 * cleared: every call writes what it reads.
 */
#define BIMAMBA_STATIC_SCRATCH_BYTES (64u << 20)
int bimamba_block_fwd_static(const bimamba_desc* desc, const bimamba_params* pf, const bimamba_params* pb,
                             const bimamba_inputs* in_f, const bimamba_inputs* in_b,
                             const float* h_in, const void* tail_in, float* h_out, void* tail_out,
                             const bimamba_tensor* out, void* hip_stream);

/* One layer of a stack: its parameters, its cached state fp32 [batch, d_inner, d_state] (NULL = zero, not committed) and its
 * conv tail, io_dtype [batch, d_conv-1, d_inner] (NULL = zeros, not committed). */
typedef struct bimamba_stack_layer {
    bimamba_params f, b;
    float* h;
    void* tail;
} bimamba_stack_layer;

/*
 * All denoising steps of a block through a stack of layers that feed each other, in one launch: for every step, layer 0 reads the
 * step's x, layer l + 1 reads layer l's output, all of them the step's z, dt, B and C; every call is bimamba_block_fwd's with
 * COMBINE_ADD, starts from its layer's cached state and tail, and the last step commits both in place.
 *   table       host array of n_layers bimamba_stack_layer, then n_steps bimamba_inputs, then n_steps * n_layers pointers: where
 *               layer l of step s (place s * n_layers + l) leaves its output, io_dtype [batch, seqlen, d_inner] contiguous, or
 *               NULL (not wanted).
 *   table_dev   a copy of it in device memory, 8-byte aligned; it stays until the work has run.
 * Outputs must not overlap any step's inputs.  Among themselves they may share memory, whole tokens apart: what a later step, or layer,
 * leaves there stays.  (A table whose steps share outputs, or whose layers share a state or a tail, is walked one step after the
 * other.)  Only for descriptors bimamba_block_stack_form answers 1 to: few enough chains that
 * a workgroup takes a few channels through the whole stack, since channels are mixed nowhere.  Nothing is allocated, no scratch is
 * used.
 */
int bimamba_block_stack(const bimamba_desc* desc, int n_layers, int n_steps, const void* table, const void* table_dev,
                        void* hip_stream);
int bimamba_block_stack_form(const bimamba_desc* desc);

/* How many of a stack's n_steps steps bimamba_block_stack takes side by side, four lanes to a chain; 0: one after the other, a row of
 * lanes to a chain (and for every descriptor that bimamba_block_stack_form answers 0 to).  For tables that share no outputs between
 * steps and no state or tail between layers; the others take their steps one after the other.  Pure host code. */
int bimamba_block_stack_side_by_side(const bimamba_desc* desc, int n_steps);

/*
 * A call's x, z, dt, B and C into buffers of the caller, in one launch: a decode loop refreshes the fixed inputs of a captured step with
 * it.  Both sides are views as for bimamba_fwd; the buffers must not overlap the sources or each other (BIMAMBA_ERR_ALIAS).
 */
int bimamba_copy_inputs(const bimamba_desc* desc, const bimamba_inputs* from, const bimamba_inputs* to, void* hip_stream);

/* Gradients with respect to the activations one direction read.  dx, dz [batch, L, d_inner] and ddt [batch, L, n_heads]
 * are views in io_dtype like the inputs (written, one rounding each); dB, dC are contiguous fp32
 * [batch, L, n_groups, d_state] device arrays (sums over the channels of a group, formed in fp32 in a fixed order;
 * overwritten, not accumulated into). */
typedef struct bimamba_input_grads {
    bimamba_tensor dx, dz, ddt;
    float* dB;
    float* dC;
} bimamba_input_grads;

/* Gradients with respect to one direction's parameters: device pointers, fp32, contiguous, shaped like bimamba_params;
 * sums over batch and tokens (overwritten, not accumulated into), formed in a fixed order: two calls on the same inputs
 * give the same bits.  dconv_b / ddt_bias may be NULL (not wanted). */
typedef struct bimamba_param_grads {
    float* dconv_w;
    float* dconv_b;
    float* dA;
    float* dD;
    float* ddt_bias;
} bimamba_param_grads;

/*
 * Gradients of bimamba_fwd (the paper trains the model, App. A.2; the backward rule is the chain rule of eqs. 4-6 in
 * the selective form, stated in csrc/bwd_kernels.h).
 *   desc, pf, pb, in_f, in_b   as for bimamba_fwd (in_b == NULL or == in_f: both directions read the same activations).
 *   dout        gradient of bimamba_fwd's out: [batch, L, d_inner] (ADD) or [batch, L, 2*d_inner] (SEPARATE), io_dtype.
 *   din_f       gradients w.r.t. in_f; with shared activations they hold the sum of both directions' contributions
 *               and din_b must be NULL.  With separate activations din_b is required.
 *   dpf, dpb    gradients w.r.t. pf and pb.  If pb == pf (tied weights) the caller adds dpb to dpf; the two must still
 *               be distinct buffers.
 *   workspace   at least bimamba_bwd_workspace_bytes(desc) bytes, 16-byte aligned.
 * Supported: the selective-scan layout, i.e. n_heads == d_inner (Delta, A, D per channel), a_kind PER_HEAD_STATE,
 * d_kind PER_CHANNEL, conv_bc 0, d_state 4, 8 or 16; every other descriptor returns BIMAMBA_ERR_UNSUPPORTED.
 * Nothing may overlap: the gradient views among themselves, the inputs, dout.  (Not checked.)
 * The call enqueues kernels only (no memset nodes), so it can be captured into a HIP graph as it is.
 */
int bimamba_bwd(const bimamba_desc* desc, const bimamba_params* pf, const bimamba_params* pb,
                const bimamba_inputs* in_f, const bimamba_inputs* in_b, const bimamba_tensor* dout,
                const bimamba_input_grads* din_f, const bimamba_input_grads* din_b,
                const bimamba_param_grads* dpf, const bimamba_param_grads* dpb,
                void* workspace, size_t workspace_bytes, void* hip_stream);

/* Workspace of bimamba_bwd: fp32 B|C rows, the state entering every chunk of 8 tokens for both directions (2 * batch *
 * L / 8 * d_inner * d_state floats), the sums at the ends of the time segments a call is cut into, 12 bytes per (batch,
 * token, channel) for the values one direction leaves for the other to add, and the per-wave partial sums of dB and dC. */
size_t bimamba_bwd_workspace_bytes(const bimamba_desc* desc);

/* Bytes of device scratch bimamba_fwd (block_variant 0) or bimamba_block_fwd (1) needs for this descriptor (0 on an invalid
 * descriptor).  The two differ where a block call is held to segments that fit BIMAMBA_STATIC_SCRATCH_BYTES; the larger of
 * them serves both.  Pure host code. */
size_t bimamba_workspace_bytes(const bimamba_desc* desc, int block_variant);

/* Number of pieces bimamba_fwd would cut the time axis into for this descriptor, each piece scanned by its own
 * workgroups and joined through a carry pass (>= 1; 0 on an invalid descriptor): the time segments of the
 * lane-per-chain kernels (1 for short calls with few chains, which one workgroup walks from end to end, in whatever
 * pieces), or the time parts of the chunked matrix-core kernels, which are 1 unless a call has so few (batch, head)
 * pairs that they would leave half of the chip empty.  1 too for such calls whose directions are added and which would have few parts:
 * they walk from both ends at once, in two launches that meet in the middle, without a carry pass (but where z or out has a token
 * stride beyond 2^24 elements, which the answer does not know of: those take the parts).  Pure host code. */
int bimamba_time_chunks(const bimamba_desc* desc);

/* ---- What stands around the mixers of a denoiser: token table, layer norm, log probabilities, clipped gradients ----
 *
 * The calls below share the rules above (host validation, caller's memory and stream, nothing allocated or kept) and these:
 * rows are (batch, token) pairs, batch * seqlen < 2^31 or what a call states (beyond it BIMAMBA_ERR_UNSUPPORTED); views read have
 * any non-negative strides (0 repeats a row), rows of a view written must lie apart from each other and from everything read
 * (BIMAMBA_ERR_ALIAS), but where a call allows the very same view; all sums, statistics and parameter gradients are fp32 or
 * wider and formed in a fixed order: the same inputs give the same bits.  Activations need be aligned to their element only.
 * No call records a memset node. */

/* Token ids [batch, seqlen] in device memory: id (b, t) at ptr + b*stride_batch + t*stride_token, 8-byte aligned. */
typedef struct bimamba_tokens {
    const int64_t* ptr;
    int64_t stride_batch;
    int64_t stride_token;
} bimamba_tokens;

/* Host struct.  vocab < 2^21, d_model <= 2^20; scale finite. */
typedef struct bimamba_embed_desc {
    uint32_t struct_size;   /* sizeof(bimamba_embed_desc), checked */
    int32_t batch;          /* >= 0 */
    int32_t seqlen;         /* >= 0 */
    int32_t d_model;
    int32_t vocab;
    int32_t table_dtype;    /* bimamba_dtype of the table (the table's gradient is fp32 whatever it is) */
    int32_t io_dtype;       /* bimamba_dtype of out and dout */
    float scale;
} bimamba_embed_desc;

/* out[b, t, :] = scale * table[id(b, t), :], one rounding; table [vocab, d_model] contiguous.  An id outside [0, vocab) gives a
 * row of zeros. */
int bimamba_embed(const bimamba_embed_desc* desc, const bimamba_tokens* tokens, const void* table, const bimamba_tensor* out,
                  void* hip_stream);

/* dtable[v, :] = scale * sum of dout[b, t, :] over the places with id v; fp32 [vocab, d_model] contiguous, every row is written
 * (rows of ids that do not occur: zeros).  Ids outside [0, vocab) count nowhere.
 * ceil(batch * seqlen / 64) * ceil(d_model / 512) < 2^25.
 *   workspace   at least bimamba_embed_bwd_workspace_bytes(desc) bytes, 16-byte aligned. */
int bimamba_embed_bwd(const bimamba_embed_desc* desc, const bimamba_tokens* tokens, const bimamba_tensor* dout, float* dtable,
                      void* workspace, size_t workspace_bytes, void* hip_stream);
size_t bimamba_embed_bwd_workspace_bytes(const bimamba_embed_desc* desc);

/* Host struct.  eps > 0. */
typedef struct bimamba_norm_desc {
    uint32_t struct_size;   /* sizeof(bimamba_norm_desc), checked */
    int32_t batch;          /* >= 0, <= 65535 */
    int32_t seqlen;         /* >= 0 */
    int32_t d_model;        /* <= 65536 */
    int32_t io_dtype;       /* bimamba_dtype of x, y, dy, dx */
    float eps;
} bimamba_norm_desc;

/* Layer norm of every row: y = (x - mean) * rstd * weight + bias, rstd = 1 / sqrt(mean((x - mean)^2) + eps).
 *   weight, bias    fp32, unit stride, or NULL (1 and 0).  weight_stride 0: one vector [d_model] for all rows; >= d_model: batch
 *                   element b has its own at + b * weight_stride (AdaLN; both may be column slices of one projection output).
 *   mean, rstd      fp32 [batch, seqlen] contiguous, or NULL (not wanted; the gradients take them). */
int bimamba_layer_norm(const bimamba_norm_desc* desc, const bimamba_tensor* x, const float* weight, const float* bias,
                       int64_t weight_stride, const bimamba_tensor* y, float* mean, float* rstd, void* hip_stream);

/* Its gradients.  With xh = (x - mean) * rstd and g = dy * weight: dx = rstd * (g - mean(g) - xh * mean(g * xh));
 * dweight = sum of dy * xh and dbias = sum of dy over the rows that share the vector: fp32 [batch, d_model] contiguous, or
 * [d_model] with weight_stride 0; NULL: not wanted.
 *   workspace   at least bimamba_layer_norm_bwd_workspace_bytes(desc, weight_stride != 0) bytes, 16-byte aligned; may be NULL if
 *               that is 0 or neither dweight nor dbias is wanted. */
int bimamba_layer_norm_bwd(const bimamba_norm_desc* desc, const bimamba_tensor* x, const float* weight, int64_t weight_stride,
                           const float* mean, const float* rstd, const bimamba_tensor* dy, const bimamba_tensor* dx,
                           float* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t bimamba_layer_norm_bwd_workspace_bytes(const bimamba_norm_desc* desc, int per_batch);

/* Host struct.  0 <= top_k <= 8, top_k <= vocab. */
typedef struct bimamba_logits_desc {
    uint32_t struct_size;   /* sizeof(bimamba_logits_desc), checked; 28, the size up to `reserved`: one without lse_rest */
    int32_t batch;          /* >= 0 */
    int32_t seqlen;         /* >= 0 */
    int32_t vocab;
    int32_t io_dtype;       /* bimamba_dtype of the logits and their gradient */
    int32_t top_k;          /* alternatives wanted per row */
    int32_t targets_only;   /* 0 or 1: rows without a target are not read (training on masked places); all they get are zeros,
                               and -1 for tokens */
    int32_t reserved;       /* 0 */
    float* lse_rest;        /* device, fp32 [batch, seqlen] contiguous, or NULL: what rounding to fp32 left of lse.  bimamba_log_probs
                               writes it (0 where lse is not finite), bimamba_log_probs_bwd reads it beside lse */
} bimamba_logits_desc;

/* What is wanted of a call's rows, device pointers, contiguous; NULL: not wanted.
 *   logp       fp32 [batch, seqlen]          log probability of the target; 0 without one (id outside [0, vocab))
 *   lse        fp32 [batch, seqlen]          log of the sum of exp(logits)
 *   entropy    fp32 [batch, seqlen]          -sum p log p
 *   top_logp   fp32 [batch, seqlen, top_k]   the largest log probabilities, in descending order
 *   top_token  int64 [batch, seqlen, top_k]  and their ids; of equal logits the lowest id comes first */
typedef struct bimamba_scores {
    float* logp;
    float* lse;
    float* entropy;
    float* top_logp;
    int64_t* top_token;
} bimamba_scores;

/*
 * Log probabilities of given tokens under softmax(logits), with the entropy and the most probable tokens of every row.
 * batch * seqlen < 2^24.
 *   logits   [batch, seqlen, vocab].  -inf is a mask: probability 0; so, beside others, is the type's lowest value, which is a number:
 *            a row of nothing but it is uniform.  A row of nothing but -inf has lse -inf, logp -inf, entropy 0, alternatives
 *            0, 1, ... with -inf.  A NaN or +inf makes a row's values NaN and its alternatives -1.
 *   targets  NULL: none (then out->logp must be NULL and targets_only 0).
 *   workspace   at least bimamba_log_probs_workspace_bytes(desc) bytes, 16-byte aligned (may be NULL if 0).
 */
int bimamba_log_probs(const bimamba_logits_desc* desc, const bimamba_tensor* logits, const bimamba_tokens* targets,
                      const bimamba_scores* out, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t bimamba_log_probs_workspace_bytes(const bimamba_logits_desc* desc);

/* Gradient for the logits: dlogits_v = dlogp * (1[v = target] - p_v) - dentropy * p_v * (log p_v + entropy), log p_v = logits_v - lse.
 *   lse, entropy      what bimamba_log_probs gave (entropy: required with dentropy).  lse is fp32, so without desc's lse_rest every p
 *                     of a row is off by up to 2^-24 |lse|, relatively; from |lse| of 2^28 on nothing is left of the sum, and a row
 *                     of equal logits has p = 1 throughout.  With lse_rest p is right whatever the logits' size.
 *   dlogp, dentropy   fp32 [batch, seqlen] contiguous; either may be NULL (0), dlogp is taken as 0 where there is no target.
 *   dlogits           may be the very view of the logits (same pointer and strides): the gradient takes their place.
 * Rows whose two gradients are 0, and rows of nothing but -inf, get zeros and are not read.  With desc's targets_only so do rows
 * without a target, whose scores are constants, whatever their dentropy (targets must then be given).  (top_k is not used.)
 * batch * seqlen * ceil(vocab / 8192) < 2^31. */
int bimamba_log_probs_bwd(const bimamba_logits_desc* desc, const bimamba_tensor* logits, const bimamba_tokens* targets,
                          const float* lse, const float* entropy, const float* dlogp, const float* dentropy,
                          const bimamba_tensor* dlogits, void* hip_stream);

/* One gradient tensor of a clipping call: count elements at `from`, contiguous; the scaled ones go to `to`, which is `from`
 * itself or memory apart from it, and in either case apart from what every other entry reads or writes: a tensor that is scaled
 * in place is listed once. */
typedef struct bimamba_grad {
    const void* from;
    void* to;
    int64_t count;
    int64_t first;          /* filled by bimamba_clip_layout */
    int32_t dtype;          /* bimamba_dtype */
    int32_t reserved;       /* 0 */
} bimamba_grad;

/* Fills `first` of a host table of n tensors.  BIMAMBA_OK, or an error: a table that bimamba_clip_grads would refuse, or one whose
 * entries meet (BIMAMBA_ERR_ALIAS; looked at here, once for a table, and not again in each bimamba_clip_grads). */
int bimamba_clip_layout(bimamba_grad* table, int n);

/*
 * Clipping by the global norm: norm = sqrt(sum of squares of all tensors), to = from * min(1, max_norm / norm).
 *   table, table_dev   host array of n tensors that bimamba_clip_layout has filled, and a copy of it in device memory, 8-byte
 *                      aligned, which stays until the work has run.
 *   max_norm           >= 0; +inf: the norm alone, gradients as they are.
 *   norm               fp32, one value on the device, or NULL.  Squares are summed in 64 bits, so they neither overflow nor vanish.
 *   workspace          at least bimamba_clip_grads_workspace_bytes(table, n) bytes, 16-byte aligned.
 * A norm that is not finite leaves the gradients as they are (`to` gets copies); the caller sees it in `norm` and skips the step.
 */
int bimamba_clip_grads(const bimamba_grad* table, int n, const void* table_dev, float max_norm, float* norm, void* workspace,
                       size_t workspace_bytes, void* hip_stream);
size_t bimamba_clip_grads_workspace_bytes(const bimamba_grad* table, int n);

/* ---- The block of a gated linear recurrence: the recurrence, the norm of its gated output, dropout into the residual stream ----
 *
 * The calls below keep the rules of the section above. */

enum bimamba_gate {
    BIMAMBA_GATE_LOG = 0,      /* g is the logarithm of the factor: a = exp(min(g, 0)), u = x */
    BIMAMBA_GATE_SIGMOID = 1   /* a = sigmoid(g + bias), u = (1 - a) * x */
};

/* Host struct. */
typedef struct bimamba_recurrence_desc {
    uint32_t struct_size;   /* sizeof(bimamba_recurrence_desc), checked */
    int32_t batch;          /* >= 0, <= 65535 */
    int32_t seqlen;         /* >= 0; above 4 tokens batch * ceil(seqlen / 64) * ceil(d_inner / 64) < 2^23 (BIMAMBA_ERR_UNSUPPORTED) */
    int32_t d_inner;        /* <= 65536 */
    int32_t io_dtype;       /* bimamba_dtype of x, g, add, y and of dy, dx, dg */
    int32_t gate;           /* bimamba_gate */
    int32_t reverse;        /* 0: tokens 0, 1, ...; 1: from a sequence's last token to its first */
} bimamba_recurrence_desc;

#define BIMAMBA_RECURRENCE_KEEP 64

/*
 * h = a h + u for every channel along the sequence, y = h + add, a mixer without state expansion: of two calls, one with `reverse`
 * that adds the other's y, comes a bidirectional one.  With h_in and h_out it goes on where an earlier call stopped: blocks, single tokens.
 *   bias      fp32 [d_inner] or NULL (0); sigmoid gates only (else BIMAMBA_ERR_UNSUPPORTED).
 *   add       [batch, seqlen, d_inner] or NULL; may be the very view y.
 *   lengths   int64 [batch] on the device or NULL: sequence b has the first lengths[b] tokens (taken into [0, seqlen]).  Tokens behind
 *             them are read into nothing; their y are zeros.
 *   h_in      fp32 [batch, d_inner], the state before a sequence's first step, or NULL (0).
 *   h_out     the same after its last step, or NULL.  May be h_in.
 *   states    fp32 [batch, ceil(seqlen / 64), d_inner] or NULL: the state before every 64th step (BIMAMBA_RECURRENCE_KEEP), counted in
 *             the order of the walk; the gradients take them.  Behind a sequence's end: its last state.
 *   workspace at least bimamba_recurrence_workspace_bytes(desc) bytes, 16-byte aligned; may be NULL if that is 0.
 * A value that is not finite makes everything not finite that its channel's walk reaches after it, up to factors whose product is 0 (a
 * factor of 0, or one that underflows): whether it reaches past those, and whether into both y and h_out, is left open.
 * All arithmetic is fp32, y is rounded once.  What a step is off by stays in the states that leave the call, and in the gradients' dh_in and dbias: its
 * own rounding, up to 2^-24, and that of a sigmoid's factor near 1, up to 2^-25 with fp32 activations and 2^-23 with bf16 ones, of the state,
 * as many times as the channel remembers tokens (bf16: 2^-13 at 700 of them; from some 20000 on more than a bf16 y loses as it is rounded).
 */
int bimamba_recurrence(const bimamba_recurrence_desc* desc, const bimamba_tensor* x, const bimamba_tensor* g, const float* bias,
                       const bimamba_tensor* add, const int64_t* lengths, const float* h_in, const bimamba_tensor* y, float* h_out,
                       float* states, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t bimamba_recurrence_workspace_bytes(const bimamba_recurrence_desc* desc);

/*
 * Its gradients (that of add is dy).  With the step's dh = dy + (a dh of the next step), the last one's from dh_out:
 *   log       dx = dh, dg = dh h' a (0 where g > 0), h' the state before the step
 *   sigmoid   dx = dh (1 - a), dg = dh (h' - x) a (1 - a)
 *   states    what bimamba_recurrence left.  bias, lengths: as there.
 *   dh_out    fp32 [batch, d_inner], the gradient of h_out, or NULL (0).
 *   dx, dg    zeros behind a sequence's end.
 *   dbias     fp32 [d_inner], the sum of dg over all tokens, or NULL; sigmoid gates only.
 *   dh_in     fp32 [batch, d_inner] or NULL.  May be dh_out.
 *   workspace at least bimamba_recurrence_bwd_workspace_bytes(desc) bytes, 16-byte aligned; may be NULL if that is 0.
 */
int bimamba_recurrence_bwd(const bimamba_recurrence_desc* desc, const bimamba_tensor* x, const bimamba_tensor* g, const float* bias,
                           const int64_t* lengths, const float* states, const bimamba_tensor* dy, const float* dh_out,
                           const bimamba_tensor* dx, const bimamba_tensor* dg, float* dbias, float* dh_in,
                           void* workspace, size_t workspace_bytes, void* hip_stream);
size_t bimamba_recurrence_bwd_workspace_bytes(const bimamba_recurrence_desc* desc);

enum bimamba_norm_act {
    BIMAMBA_ACT_NONE = 0,
    BIMAMBA_ACT_SILU = 1,          /* y = SiLU(norm(x)) */
    BIMAMBA_ACT_GATE_BEFORE = 2,   /* y = norm(x * SiLU(z)) */
    BIMAMBA_ACT_GATE_AFTER = 3     /* y = norm(x) * SiLU(z) */
};

/* Host struct.  d_inner is a multiple of groups; at most 8192 channels a group. */
typedef struct bimamba_group_norm_desc {
    uint32_t struct_size;   /* sizeof(bimamba_group_norm_desc), checked */
    int32_t batch;          /* >= 0 */
    int32_t seqlen;         /* >= 0 */
    int32_t d_inner;        /* <= 65536 */
    int32_t groups;         /* >= 1 */
    int32_t io_dtype;       /* bimamba_dtype of x, z, y and of dy, dx, dz */
    int32_t act;            /* bimamba_norm_act */
    int32_t centred;        /* 0: root mean square; 1: the mean is taken off first */
    float eps;              /* > 0 */
} bimamba_group_norm_desc;

/* The norm of every token's groups of channels (neighbours each): with u = x, or x * SiLU(z), v = (u - mean) * rstd * weight + bias,
 * rstd = 1 / sqrt(mean((u - mean)^2) + eps), mean 0 unless centred; y = v, SiLU(v) or v * SiLU(z).
 *   z               the gate's input; gates only (else it must be NULL: BIMAMBA_ERR_UNSUPPORTED).
 *   weight, bias    fp32 [d_inner] or NULL (1 and 0).
 *   mean, rstd      fp32 [batch, seqlen, groups] or NULL (not wanted; the gradients take them); mean: centred only. */
int bimamba_group_norm(const bimamba_group_norm_desc* desc, const bimamba_tensor* x, const bimamba_tensor* z, const float* weight,
                       const float* bias, const bimamba_tensor* y, float* mean, float* rstd, void* hip_stream);

/* Its gradients.  With xh = (u - mean) * rstd and dv = dy, dy * SiLU'(v) or dy * SiLU(z): dweight = sum of dv * xh and dbias = sum of dv
 * over all tokens, fp32 [d_inner], NULL: not wanted; with k = dv * weight, du = rstd * (k - mean(k) - xh * mean(k * xh)) (mean(k):
 * centred only); dx = du or du * SiLU(z); dz = dy * v * SiLU'(z) or du * x * SiLU'(z).
 *   workspace   at least bimamba_group_norm_bwd_workspace_bytes(desc) bytes, 16-byte aligned; may be NULL if that is 0 or neither dweight
 *               nor dbias is wanted. */
int bimamba_group_norm_bwd(const bimamba_group_norm_desc* desc, const bimamba_tensor* x, const bimamba_tensor* z, const float* weight,
                           const float* bias, const float* mean, const float* rstd, const bimamba_tensor* dy, const bimamba_tensor* dx,
                           const bimamba_tensor* dz, float* dweight, float* dbias, void* workspace, size_t workspace_bytes,
                           void* hip_stream);
size_t bimamba_group_norm_bwd_workspace_bytes(const bimamba_group_norm_desc* desc);

/* Host struct.  d_model <= 2^20, 0 <= site < 2^15. */
typedef struct bimamba_dropout_desc {
    uint32_t struct_size;   /* sizeof(bimamba_dropout_desc), checked */
    int32_t batch;          /* >= 0, <= 65535 */
    int32_t seqlen;         /* >= 0 */
    int32_t d_model;
    int32_t io_dtype;       /* bimamba_dtype of x, residual, out and of dout, dx */
    int32_t site;           /* which of a model's dropouts it is: sites have masks of their own under one key */
    float p;                /* share that is dropped, in [0, 1]; taken as round(65536 p) / 65536 */
} bimamba_dropout_desc;

/*
 * out = residual + gate * dropout(x).  No mask is stored: value (b, t, c) is kept where its 16 random bits are at least T = round(65536 p),
 * and multiplied by 65536 / (65536 - T); T = 65536 keeps nothing.  Its bits are half c % 8 (the low half of a word first) of the
 * four words that Philox4x32 with ten rounds (Salmon et al., 2011) makes of the counter (b * seqlen + t, c / 8 + site * 2^17, low and
 * high word of the offset) under the seed as its key.
 *   key        int64 [2] on the device: seed, offset.  A program moves the offset between steps, in a captured graph too.
 *   gate       fp32, unit stride, or NULL (1).  gate_stride 0: one vector [d_model]; >= d_model: batch element b has its own at
 *              gate + b * gate_stride.
 *   residual   or NULL (0); may be the very view out.
 * What is dropped is not read into the result: a NaN there leaves the residual as it is.
 */
int bimamba_dropout_add(const bimamba_dropout_desc* desc, const int64_t* key, const bimamba_tensor* x, const float* gate,
                        int64_t gate_stride, const bimamba_tensor* residual, const bimamba_tensor* out, void* hip_stream);

/* Its gradients (the residual's is dout): dx = gate * keep * dout / (1 - p), and dgate = the sum of keep * x * dout / (1 - p) over the
 * tokens that share the vector, fp32 [batch, d_model] contiguous, or [d_model] with gate_stride 0; NULL: not wanted, x may then be NULL too.
 *   dx          may be the very view dout.
 *   workspace   at least bimamba_dropout_add_bwd_workspace_bytes(desc, gate_stride != 0) bytes, 16-byte aligned; may be NULL if that is 0
 *               or dgate is not wanted. */
int bimamba_dropout_add_bwd(const bimamba_dropout_desc* desc, const int64_t* key, const bimamba_tensor* x, const float* gate,
                            int64_t gate_stride, const bimamba_tensor* dout, const bimamba_tensor* dx, float* dgate, void* workspace,
                            size_t workspace_bytes, void* hip_stream);
size_t bimamba_dropout_add_bwd_workspace_bytes(const bimamba_dropout_desc* desc, int per_batch);

/* Benchmark diagnostics: arm a one-shot probe on the calling host thread.  The next bimamba_fwd or
 * bimamba_block_fwd made by this thread records ev_start immediately before and ev_stop immediately after its
 * scan-and-combine kernel (on the chunked matrix-core path: around its two launches, one per direction; never the
 * B|C preparation, segment summary or tail kernels) on that call's stream, then disarms.  Both are hipEvent_t created by the caller with timing enabled; NULL, NULL disarms.  This thread-local
 * pair is the only state the library keeps between calls. */
void bimamba_profile_next_call(void* ev_start, void* ev_stop);

/* Static, NUL-terminated description of a status code. */
const char* bimamba_status_string(int status);

/* BIMAMBA_VERSION the library was built from. */
int bimamba_version(void);

#ifdef __cplusplus
}
#endif
#endif /* BIMAMBA_H */
