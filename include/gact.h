/*
 * gact.h -- C ABI of the MI355X (gfx950) activation compressor / decompressor
 * of GACT (arXiv 2206.11357) and its host-side bit allocator.
 *
 * What the calls compute
 *   The paper's compressor Q is a per-group stochastic-rounding quantizer
 *   (Sec. 5: quantisation per group; App. A.4: transform
 *   T(h_j) = (2^b-1)(h_j - min h)/(max h - min h), round up with probability
 *   T - floor(T), otherwise down, and map back with the inverse of T).  A
 *   context tensor is a flattened vector (Sec. 3.1); it is cut into groups of
 *   `group_size` consecutive elements, the last group may be shorter.
 *   Per-tensor bit widths b_l come from Eq. (ilp) of Sec. 4.1,
 *   min sum_l c_l S(b_l) s.t. sum_l b_l D_l <= budget, S(b) = (2^b-1)^-2.
 *
 * Arithmetic (bit-exact contract)
 *   IEEE binary32, round to nearest even, every operation rounded on its own
 *   (no fused multiply-add where it would change a result):
 *     mn = min, mx = max over the group;  mn = mn + 0.0f (so -0 is stored as +0)
 *     range = mx - mn;  B = 2^bits - 1
 *     range >= 2^-100 :  inv = B / range,  step = range / B
 *     otherwise       :  inv = 0,          step = 0        (constant group)
 *     t = (x - mn) * inv;  q = floor(t) + (u < t - floor(t));  q = min(q, B)
 *     y = q * step + mn                  (decompress; bf16 output rounds y RNE)
 *   Rounding noise u for element i of a tensor compressed with `seed`:
 *   Philox4x32-10 (Salmon et al., SC'11), key = (low, high 32 bits of seed),
 *   counter = (low, high 32 bits of i/8, 0, 0).  The four output words hold
 *   eight 16-bit slots, low half first; element i takes slot i%8 and
 *   u = (slot + 0.5) / 65536.  (For a shard, i counts from the descriptor's
 *   index_base.)  The stream is a function of (seed, i) only, so
 *   results never depend on launch shape or on single- vs multi-tensor calls,
 *   and the same seed replays the same compression (Alg. 1 of the paper relies
 *   on replayable per-tensor seeds).
 *
 * Layouts
 *   packed : linear bit string, element i in bits [i*bits, (i+1)*bits), bit k
 *            of the string is bit k%8 of byte k/8 (little-endian, LSB first).
 *            gact_packed_bytes(n, bits) bytes; all pad bits are written as 0.
 *   gmin   : float[gact_num_groups]  group minimum.
 *   gscale : float[gact_num_groups]  dequantisation step, range / (2^bits-1).
 *
 * Memory and ownership
 *   Pointers named d_* are DEVICE pointers owned by the caller; h_* are HOST
 *   pointers.  The library allocates nothing, frees nothing and keeps no
 *   pointer after a call returns.  d_x, d_y, d_packed and the multi-tensor
 *   workspace must be 16-byte aligned; d_gmin / d_gscale 4-byte aligned.
 *   Device calls enqueue work on `stream` (a hipStream_t passed as void*;
 *   NULL is the default stream) and return without waiting for it.
 *
 * Errors
 *   Every call returns GACT_OK or a negative code; on error nothing has been
 *   enqueued.  Inputs must be finite with max - min finite; NaN / Inf give
 *   unspecified values but never an out-of-bounds access.
 */
#ifndef GACT_H
#define GACT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { GACT_F32 = 0, GACT_BF16 = 1 } gact_dtype;

/* Bit width that means "leave this tensor uncompressed" in the allocator's
 * level sets and in multi-tensor descriptors. */
#define GACT_BITS_UNCOMPRESSED 32

enum {
    GACT_OK       =  0,
    GACT_E_ARG    = -1,  /* null pointer, n < 0, misaligned pointer, bad dtype, L < 0,
                            negative / non-finite sensitivity or numel, workspace too small */
    GACT_E_BITS   = -2,  /* bits not in {1,2,4,8} */
    GACT_E_GROUP  = -3,  /* group_size not a multiple of 32 in [32, 1024] */
    GACT_E_BUDGET = -4,  /* avg_bit_budget < 1 or NaN: no feasible scheme */
    GACT_E_HIP    = -5,  /* the HIP runtime refused the launch or copy */
    GACT_E_CAPTURE = -6, /* the stream is being captured into a HIP graph and this call
                            would have to upload a table from host memory (the two
                            reductions over buffer lists: whether they would or not) */
    GACT_E_SCRATCH = -7  /* gact_compress_footprint_noalloc: the tensor needs more than the
                            library's static scratch area */
};

/* ceil(n / group_size); 0 when n <= 0 or group_size <= 0. */
size_t gact_num_groups(int64_t n, int group_size);

/* ceil(n * bits / 8) rounded up to a multiple of 16; 0 when n <= 0. */
size_t gact_packed_bytes(int64_t n, int bits);

/* Human-readable name of an error code (static string). */
const char *gact_error_string(int code);

/*
 * Compressor (forward pass; App. A.4 applied per group, Sec. 5).
 *   d_x      in   n elements of `dtype`, contiguous, not modified
 *   d_packed out  gact_packed_bytes(n, bits) bytes
 *   d_gmin   out  gact_num_groups(n, group_size) floats
 *   d_gscale out  same count
 * n == 0 is GACT_OK and launches nothing.
 */
int gact_compress(const void *d_x, gact_dtype dtype, int64_t n, int group_size,
                  int bits, uint64_t seed, void *d_packed, float *d_gmin,
                  float *d_gscale, void *stream);

/*
 * Decompressor (backward pass; inverse transform of App. A.4).
 *   d_y out  n elements of `dtype`.  Must not overlap the inputs.
 */
int gact_decompress(const void *d_packed, const float *d_gmin,
                    const float *d_gscale, int64_t n, int group_size, int bits,
                    void *d_y, gact_dtype dtype, void *stream);

/*
 * Multi-tensor launches: the many saved tensors of one iteration (the paper's
 * hook compresses every saved tensor of every operator, Sec. 5) in one launch
 * per direction.  Each descriptor carries its own element count, dtype, bits
 * and seed (the per-tensor seeds r_l of Alg. 1).  The result for each tensor
 * is byte-identical to the single-tensor call with the same arguments.
 *
 *   h_descs          host array of L descriptors; device pointers inside.
 *                    compress reads x and writes packed/gmin/gscale (y unused);
 *                    decompress reads packed/gmin/gscale and writes y (x unused).
 *   d_workspace      device scratch of at least gact_multi_workspace_bytes(L)
 *                    bytes, 16-byte aligned.  With more than 64 non-empty
 *                    tensors it holds the launch table until the enqueued
 *                    kernel has run, so it must not be reused for a different
 *                    table before then; smaller tables travel in the kernel
 *                    arguments and leave it untouched.
 * A table in the workspace is uploaded with a stream-ordered copy from host
 * memory the call owns; h_descs may be reused as soon as the call returns.
 * HIP graphs: with at most 64 non-empty tensors a call enqueues exactly one
 * kernel and can be captured (pointers, sizes, bits and seeds are baked into
 * the node).  A larger table needs an upload from host memory the call owns,
 * which a graph could not replay: on a capturing stream such a call enqueues
 * nothing and returns GACT_E_CAPTURE -- capture those sets in slices of 64.
 * Shards: the noise of element i is a function of (seed, index_base + i) only,
 * so a tensor cut at multiples of the group size and compressed piece by piece
 * (on one GPU or on several), each piece with the tensor's seed and its own
 * offset as index_base, gives pieces whose packed strings, minima and steps
 * concatenate to the result for the whole tensor.  index_base must be a
 * non-negative multiple of 8 (GACT_E_ARG otherwise); decompress ignores it.
 * A descriptor with bits == GACT_BITS_UNCOMPRESSED is skipped by both calls:
 * the allocator left that tensor at full precision and the caller keeps it.
 * L == 0, or all n == 0, is GACT_OK and launches nothing.
 */
typedef struct {
    const void *x;
    void       *packed;
    float      *gmin;
    float      *gscale;
    void       *y;
    int64_t     n;
    uint64_t    seed;
    int32_t     bits;
    int32_t     dtype;     /* gact_dtype */
    int64_t     index_base; /* compress: index of x[0] in the noise stream (see below); 0 for a whole tensor */
} gact_tensor_desc;

size_t gact_multi_workspace_bytes(int L);

int gact_compress_multi(const gact_tensor_desc *h_descs, int L, int group_size,
                        void *d_workspace, size_t workspace_bytes, void *stream);

int gact_decompress_multi(const gact_tensor_desc *h_descs, int L, int group_size,
                          void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Sensitivity of one context tensor (Alg. 1, Sec. 4.2).  g0 and g1 are the
 * gradients of two iterations that differ only in the seed of tensor l's
 * compressor, each a list of K parameter buffers; the call computes
 *     c_l = 1/2 * sum_k ||g0_k - g1_k||^2 / S(bits),   S(b) = (2^b-1)^-2,
 * `bits` being the width tensor l was compressed with, accumulated in binary64
 * in a fixed order (the result does not depend on scheduling, nor on what other
 * streams run meanwhile).
 *   h_pairs      host array of K buffer pairs; device pointers inside, 16-byte
 *                aligned, both buffers of a pair have n elements of `dtype`.
 *   d_out        device double[1], receives c_l when the stream reaches it.
 *   d_workspace  device scratch, >= gact_reduce_workspace_bytes(K, sum of n),
 *                16-byte aligned; in use until the enqueued kernels have run.
 *                Two calls that share a workspace must not overlap in time: their
 *                results are then unspecified (a sum of either's parts, a NaN),
 *                but both end.
 * K == 0 or all n == 0 writes 0.
 * HIP graphs: this call and gact_grad_stats_update return GACT_E_CAPTURE, with
 * nothing enqueued, on a stream that is being captured.  A list of more than
 * 104 non-empty buffers needs its table uploaded from host memory the call
 * owns, which a graph could not replay; shorter lists travel in the kernel
 * arguments and are refused all the same, so that what a caller can capture
 * does not depend on how many of its buffers happen to be empty.
 */
typedef struct {
    const void *g0;
    const void *g1;
    int64_t     n;
    int32_t     dtype;     /* gact_dtype */
    int32_t     reserved;
} gact_grad_pair;

size_t gact_reduce_workspace_bytes(int K, int64_t total_elems);

int gact_sensitivity(const gact_grad_pair *h_pairs, int K, int bits, double *d_out,
                     void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Running gradient statistics for the a-posteriori alert of Sec. 4.2, which
 * needs the variance of the gradient and obtains it from a running mean kept
 * over the iterations.  Step t >= 1 over K parameter buffers, binary32 per element:
 *     mean <- mean + (g - mean) * rt,    rt = (float)(1 / t),
 * and, in binary64, d_out[0] = sum g^2, d_out[1] = sum mean_new^2.  With the
 * caller's running average s_t of d_out[0], Var[g] ~ s_t - d_out[1].
 *   mean   device float[n] per buffer, read and written in place (start at 0).
 */
typedef struct {
    const void *g;
    float      *mean;
    int64_t     n;
    int32_t     dtype;     /* gact_dtype of g */
    int32_t     reserved;
} gact_grad_stat;

int gact_grad_stats_update(const gact_grad_stat *h_stats, int K, int64_t t, double *d_out,
                           void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Footprint of a tensor for duplicate detection (Sec. 5.2: a tensor saved by
 * several operators is recognised by its data pointer, sampled points and its
 * sum, and compressed once).  One read of the tensor:
 *     d_out[0]     = sum of all elements, binary64, fixed order
 *     d_out[1 + j] = element floor(j * n / n_samples), j < n_samples <= 32768
 *   d_workspace  >= gact_reduce_workspace_bytes(1, n) bytes, 16-byte aligned.
 * n == 0 writes zeros.
 */
int gact_footprint(const void *d_x, gact_dtype dtype, int64_t n, int n_samples, double *d_out,
                   void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Compressor and footprint from one read of the tensor: the sum is taken in
 * the pass that computes the group statistics (Sec. 5.2 names the footprint,
 * App. A.4 the statistics).  Arguments and results of gact_compress, plus
 *   d_footprint  out  double[1 + n_samples], as gact_footprint defines it
 *                     (the sum is accumulated in another fixed order, so it
 *                     may differ from gact_footprint's in the last bits)
 *   d_workspace       >= gact_compress_footprint_workspace_bytes(n, group_size)
 *                     bytes, 16-byte aligned, in use until the kernels have run
 *                     (calls that share one: as for gact_sensitivity)
 * A caller that finds the footprint among tensors it already holds drops the
 * new compressed copy and keeps the old one.  n == 0 writes zeros.
 */
size_t gact_compress_footprint_workspace_bytes(int64_t n, int group_size);
int gact_compress_footprint(const void *d_x, gact_dtype dtype, int64_t n, int group_size,
                            int bits, uint64_t seed, void *d_packed, float *d_gmin,
                            float *d_gscale, int n_samples, double *d_footprint,
                            void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Copy of nbytes between buffers a kernel can address -- device memory, or host
 * memory that is pinned and mapped (hipHostMalloc) -- by a kernel of
 * `workgroups` workgroups (1..1024), enqueued on `stream`.  For the swap of
 * compressed activations to the host that Sec. 5.3 runs on a stream of its own
 * next to the forward pass: a few workgroups keep PCIe busy and leave the rest
 * of the GPU to the model, which the runtime's own device-to-host copy kernel
 * does not.  dst and src 16-byte aligned and not overlapping.  A pointer that
 * no kernel may touch (ordinary host memory) returns GACT_E_ARG, nothing is
 * enqueued.
 */
int gact_copy_bounded(void *dst, const void *src, size_t nbytes, int workgroups, void *stream);

/*
 * gact_compress_footprint for callers that cannot allocate device memory and
 * so cannot bring a workspace: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  The kernel's partial sums go to a
 * scratch area of GACT_NOALLOC_SCRATCH_BYTES that is part of the library's
 * device image (each GPU the library runs on holds one copy until the process
 * ends); the call allocates and frees nothing.  Same arguments, results and
 * error codes as gact_compress_footprint without the workspace pair; results
 * are byte-identical to that call's.
 *   Limit: room for one 8-byte partial per tile of 2048 elements (44 * 32 ...
 *   63 * 32 elements when group_size / 32 is not a power of two), i.e. up to
 *   536,870,912 elements for power-of-two group sizes; the kernel writes one per
 *   four tiles.  A larger n returns GACT_E_SCRATCH and enqueues nothing.
 *   All calls on one GPU share that GPU's area: two calls whose kernels may
 *   overlap in time (different streams, or graph launches in flight together)
 *   race on it and must be ordered by the caller.  The area keeps the last
 *   call's contents; nothing in it has to start at zero, because every partial
 *   a call reads was written by that call's own compress kernel.
 */
#define GACT_NOALLOC_SCRATCH_BYTES (2u << 20)
int gact_compress_footprint_noalloc(const void *d_x, gact_dtype dtype, int64_t n, int group_size,
                                    int bits, uint64_t seed, void *d_packed, float *d_gmin,
                                    float *d_gscale, int n_samples, double *d_footprint,
                                    void *stream);

/*
 * Global norm of a list of gradient buffers, and clipping by it.
 *     norm = sqrt(sum g^2)  (GACT_NORM_2)   or   max |g|  (GACT_NORM_INF), over all buffers together,
 *     out  = g * min(1, max_norm / (norm + 1e-6)),   from binary64 rounded to nearest, a bf16 result by way of binary32
 *                                                    (off by half a step of bf16 and 2^-24 of the value, at most),
 * the squares added in binary64 in an order that depends on the list's sizes, types and alignments only, the same in every call.  A
 * NaN among the gradients gives a NaN norm and NaN outputs; an infinity gives an infinite norm and outputs 0 (NaN at its place).
 *   gact_grad_norm     d_norm receives the norm
 *   gact_grad_clip     the same, and the scaled gradients in two launches
 *   gact_grad_clip_by  scales by the norm in d_norm: one that several ranks have agreed on, or the square root
 *                      of gact_grad_stats_update's d_out[0]
 *   h_bufs       host array of K buffers of any alignment that their type has; g and out of n elements of `dtype`.
 *                out may be g (then nothing is written where nothing has to be scaled); otherwise no output may
 *                overlap an input, and no two outputs overlap (GACT_E_ARG): a buffer listed twice is refused
 *                by the calls that scale.  gact_grad_norm ignores out and counts a buffer as often as it is listed.
 *   max_norm     finite, >= 0
 *   d_norm       device double[1]
 *   d_workspace  device scratch, >= gact_grad_norm_workspace_bytes(K), 16-byte aligned; in use until the enqueued
 *                kernels have run.  Calls that share one must not overlap in time.
 * K == 0 or all n == 0 writes the norm 0.
 * HIP graphs: all three calls can be captured, whatever K: a list of more than 136 non-empty buffers, whose table is
 * uploaded otherwise, travels in the arguments of small kernels of its own then.  A replay uses the pointers, sizes
 * and max_norm of the captured call and its workspace.
 */
typedef enum { GACT_NORM_2 = 0, GACT_NORM_INF = 1 } gact_norm_kind;

typedef struct {
    const void *g;
    void       *out;
    int64_t     n;
    int32_t     dtype;     /* gact_dtype of g and out */
    int32_t     reserved;
} gact_grad_buf;

size_t gact_grad_norm_workspace_bytes(int K);

int gact_grad_norm(const gact_grad_buf *h_bufs, int K, int kind, double *d_norm, void *d_workspace,
                   size_t workspace_bytes, void *stream);

int gact_grad_clip(const gact_grad_buf *h_bufs, int K, int kind, double max_norm, double *d_norm,
                   void *d_workspace, size_t workspace_bytes, void *stream);

int gact_grad_clip_by(const gact_grad_buf *h_bufs, int K, double max_norm, const double *d_norm,
                      void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Norms of queries and keys for each head with the position rotation in the same pass, whose context (x, the queries
 * or keys before the norm) can leave the same pass compressed, and the gradients, taken from the compressed
 * context without decompressing it to memory.  A tensor is [batch, tokens, heads, head_dim], its heads' elements
 * consecutive, every other stride its own.  For each head of each token
 *     r = 1 / sqrt(mean x^2 + eps),   n = x * r * w,
 *     y_a = n_a * cos - n_b * sin,   y_b = n_b * cos + n_a * sin
 * for the rot_dim / 2 pairs (a, b) of its first rot_dim elements, (i, i + rot_dim/2) or, `interleaved`,
 * (2i, 2i + 1); y = n from rot_dim on.  Backward, with dn = dy rotated back,
 *     dx = r * (dn * w - x * r^2 * mean(dn * w * x)),   dw = sum over heads and tokens of dn * x * r.
 * Arithmetic in binary32 (the squares of x are added in it: |x| < 2^59), dw's sums over blocks in binary64 and in a fixed
 * order; outputs rounded once.  A head's values reach no other head's.
 *
 * Context.  With bits in {1, 2, 4, 8} the forward pass writes what gact_compress gives for x laid out
 * contiguously as [batch, tokens, heads, head_dim] with the same group_size, bits and seed, byte for byte, and the backward
 * pass uses codes * step + minimum (in binary32, not rounded to the tensor's type) for x.  r is not taken from these:
 * the forward pass leaves it in rstd, so that dw is linear in the compressed x and stays unbiased.  With
 * GACT_BITS_UNCOMPRESSED nothing is compressed and the backward pass reads x.
 *
 *   h_parts      host array of 1 or 2 tensors (queries and keys), which go into one launch where their bits agree.
 *     forward:   reads x; writes y, rstd (batch * tokens * heads floats; NULL without a backward pass, only with
 *                bits == GACT_BITS_UNCOMPRESSED) and, compressing, packed (16-byte aligned), gmin and gscale.  y may be x
 *                itself with x's strides.
 *     backward:  reads dy, rstd and packed, gmin, gscale (compressed) or x; writes dx and, where dw is not NULL, dw.
 *                dx may be dy itself with dy's strides.
 *     Nothing else may overlap an output.  GACT_E_ARG for what pointers and strides show of it: a buffer given twice, in
 *     place with other strides, an output's rows that share memory (each stride of an axis longer than 1 has to pass what
 *     the smaller ones span).
 *     w, dw      head_dim weights and their gradients, of w_dtype; w NULL: no weights (dw must be NULL)
 *     strides    in elements: batch, token, head
 *     heads      may differ between the parts
 *   h_rotation   what the parts share:
 *     cos, sin   tables [n_positions, rot_dim / 2] in binary32; unused with rot_dim 0
 *     positions  device int64 [batch * tokens], or NULL: a token's place in its sequence.  A token whose position is
 *                outside [0, n_positions) gets NaN in its rotated elements (and in the gradients they reach); nothing
 *                is read outside the tables.
 *     head_dim   a multiple of 8 in [8, 512];  rot_dim a multiple of 16 in [0, head_dim]
 *     group_size of a context: a power of two in [32, 512] that divides head_dim, or a multiple of 32 that is head_dim *
 *                1, 2, 4, ... , at most 64 lanes of eight elements (a head occupies head_dim / 8 lanes rounded up to a
 *                power of two); heads * head_dim must be a multiple of it.  GACT_E_GROUP otherwise: gact_compress takes
 *                such a tensor.
 *   batch * tokens * heads must be below 2^31.
 *   d_workspace  backward: device scratch, >= gact_head_norm_rotate_workspace_bytes(head_dim), 16-byte aligned, in use
 *                until the enqueued kernels have run; calls that share one must not overlap in time.  Not used (NULL) when
 *                no dw is asked for.
 * An empty tensor (batch or tokens 0) is GACT_OK; its dw is 0.  Both calls can be captured into a HIP graph.
 */
typedef struct {
    const void *x;
    void       *y;
    const void *dy;
    void       *dx;
    const void *w;
    void       *dw;
    float      *rstd;
    void       *packed;
    float      *gmin;
    float      *gscale;
    int64_t     x_stride[3];
    int64_t     y_stride[3];
    int64_t     dy_stride[3];
    int64_t     dx_stride[3];
    uint64_t    seed;
    int32_t     heads;
    int32_t     bits;
} gact_heads;

typedef struct {
    int64_t        batch;
    int64_t        tokens;
    const float   *cos;
    const float   *sin;
    const int64_t *positions;
    int64_t        n_positions;
    int32_t        head_dim;
    int32_t        rot_dim;
    int32_t        interleaved;
    int32_t        dtype;       /* gact_dtype of x, y, dy, dx */
    int32_t        w_dtype;     /* gact_dtype of w, dw */
    int32_t        group_size;  /* of the contexts */
    float          eps;         /* a normal number > 0; forward only */
    int32_t        reserved;
} gact_rotation;

size_t gact_head_norm_rotate_workspace_bytes(int head_dim);

int gact_head_norm_rotate(const gact_heads *h_parts, int n_parts, const gact_rotation *h_rotation, void *stream);

int gact_head_norm_rotate_backward(const gact_heads *h_parts, int n_parts, const gact_rotation *h_rotation,
                                   void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Group normalisation with an activation over a channels-last map, [batch, pixels, channels] with a pixel's channels
 * consecutive and every other stride its own, whose context (x) can leave the same pass compressed, and the gradients,
 * taken from the compressed context without decompressing it to memory.  The channels lie in `groups` groups of
 * D = channels / groups; over the M = pixels * D elements of a group of a sample
 *     m = mean x,   r = 1 / sqrt(mean (x - m)^2 + eps),   n = (x - m) * r,   z = n * w + b,   y = act(z),
 * act(z) = z (GACT_ACT_NONE) or z / (1 + exp(-z)) (GACT_ACT_SILU).  Backward, n from the forward pass's m and r,
 *     dz = dy * act'(z),  g = dz * w,  dx = r * (g - mean g - n * mean(g * n)),  dw = sum of dz * n,  db = sum of dz.
 * Arithmetic in binary32.  Sums over what a wavefront holds of a group (a workgroup, where the group is too large for one) in
 * binary32, of these in binary64, m and r rounded once from there; a sample's part of dw and db is rounded to binary32.  The order
 * depends on sizes, type, width and activation only, so that every call gives the same.  Outputs are rounded once.  Samples reach
 * each other in dw and db only.
 *
 * Context.  With bits in {1, 2, 4, 8} the forward pass writes what gact_compress gives for x laid out contiguously with
 * the same group_size, bits and seed, byte for byte, and the backward pass uses codes * step + minimum (in
 * binary32, not rounded to x's type) for x in n.  m and r are not taken from these: the forward pass leaves them in mean and
 * rstd.  With GACT_BITS_UNCOMPRESSED nothing is compressed and the backward pass reads x.
 *
 *   forward    reads x; writes y, mean and rstd (batch * groups floats each; both NULL: not wanted, only with bits ==
 *              GACT_BITS_UNCOMPRESSED) and, compressing, packed (16-byte aligned), gmin and gscale.  y may be x itself with x's
 *              strides.
 *   backward   reads dy, mean, rstd and packed, gmin, gscale (compressed) or x; writes dx and, where they are not NULL, dw
 *              and db.  dx may be dy itself with dy's strides.
 *   Nothing else may overlap an output.  GACT_E_ARG for what pointers and strides show of it: a buffer given twice, in place
 *   with other strides, an output's pixels that share memory.
 *   w, b       weights and shifts of w_dtype, one a channel; NULL: ones, zeros (dw, db must be NULL then)
 *   strides    in elements: sample, pixel
 *   channels   a multiple of 8 and of groups;  group_size of a context: 32, 64, 128, 256 or 512 (GACT_E_GROUP otherwise:
 *              gact_compress takes such a tensor)
 *   batch * pixels * channels must be below 2^34, batch * pixels below 2^31, batch * channels below 2^30 (below 2^24 where a group of
 *   a sample has more than 65536 elements or so: GACT_E_ARG if a launch would pass 2^32 threads).
 *   d_workspace  device scratch, >= gact_group_norm_workspace_bytes(...) of the same sizes, dtype and pass (which may be 0),
 *              16-byte aligned, in use until the enqueued kernels have run; calls that share one must not overlap in time.
 * An empty tensor (batch or pixels 0) is GACT_OK; its dw and db are 0.  Both calls can be captured into a HIP graph.
 */
typedef enum { GACT_ACT_NONE = 0, GACT_ACT_SILU = 1 } gact_activation;

typedef struct {
    const void *x;
    void       *y;
    const void *dy;
    void       *dx;
    const void *w;
    const void *b;
    void       *dw;
    void       *db;
    float      *mean;
    float      *rstd;
    void       *packed;
    float      *gmin;
    float      *gscale;
    int64_t     x_stride[2];
    int64_t     y_stride[2];
    int64_t     dy_stride[2];
    int64_t     dx_stride[2];
    int64_t     batch;
    int64_t     pixels;
    uint64_t    seed;
    int32_t     channels;
    int32_t     groups;
    int32_t     act;         /* gact_activation */
    int32_t     dtype;       /* gact_dtype of x, y, dy, dx */
    int32_t     w_dtype;     /* gact_dtype of w, b, dw, db */
    int32_t     bits;
    int32_t     group_size;  /* of the context */
    float       eps;         /* a normal number > 0; forward only */
} gact_channel_norm;

size_t gact_group_norm_workspace_bytes(int64_t batch, int64_t pixels, int channels, int groups, gact_dtype dtype,
                                       int backward);

int gact_group_norm(const gact_channel_norm *h_norm, void *d_workspace, size_t workspace_bytes, void *stream);

int gact_group_norm_backward(const gact_channel_norm *h_norm, void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Weight gradient of a linear layer y = x W^T + b from the compressed context of its input, which is not decompressed
 * to memory:
 *     dW[n, k] = sum over t of dy[t, n] * x^[t, k],      db[n] = sum over t of dy[t, n],
 * x^ being what gact_decompress gives of the context in dy's type (x laid out contiguously as [tokens, in_features];
 * groups may pass from row to row).  Sums in binary32, over blocks and splits of the tokens in a fixed order, the same
 * in every call of the same sizes and types; outputs rounded once.
 *   dy           [tokens, out_features] of dtype, its rows' elements consecutive, dy_stride elements from row to row (any value,
 *                0 too: a gradient that all tokens share), aligned as its type
 *   packed, gmin, gscale, group_size, bits   as gact_compress has left them
 *   dw           out  [out_features, in_features], contiguous, of w_dtype
 *   db           out  [out_features] of w_dtype, or NULL: not wanted.  Outputs overlap nothing.
 *   d_workspace  device scratch, >= gact_linear_weight_grad_workspace_bytes(...) bytes of the same sizes (which may be 0),
 *                16-byte aligned, in use until the enqueued kernels have run; calls that share one must not overlap in time.
 * tokens == 0 writes zeros; out_features == 0 or in_features == 0 is GACT_OK and writes nothing but db.  tokens must
 * be below 2^31, out_features below 2^28, in_features below 2^22, tokens * in_features and out_features * in_features
 * below 2^34.  With dtype binary32, each product is exact to 2^-24 of itself, of values taken apart into bfloat16, whose least
 * number leaves 2^-134 of an element at most; an element of dW whose sum is not finite that way (infinities, NaN, elements from
 * 2^128 - 2^119 on) is added again in binary32, at the cost of a pass over its tokens.  An infinity or NaN in a row of
 * dy reaches that row's columns of dW (rows of x^ times it), in a group's minimum or step the elements of that
 * group.  Can be captured into a HIP graph.
 */
typedef struct {
    const void  *dy;
    const void  *packed;
    const float *gmin;
    const float *gscale;
    void        *dw;
    void        *db;
    int64_t      dy_stride;
    int64_t      tokens;
    int64_t      out_features;
    int64_t      in_features;
    int32_t      dtype;       /* gact_dtype of dy */
    int32_t      w_dtype;     /* gact_dtype of dw, db */
    int32_t      group_size;
    int32_t      bits;
} gact_linear_grad;

size_t gact_linear_weight_grad_workspace_bytes(int64_t tokens, int64_t out_features, int64_t in_features,
                                               gact_dtype dtype);

int gact_linear_weight_grad(const gact_linear_grad *h_grad, void *d_workspace, size_t workspace_bytes, void *stream);

/*
 * Variance alert (host only): V(b) = sum_l c_l S(b_l) (Thm. 2) against the
 * gradient variance.  Writes V / grad_var to *h_ratio (may be NULL) and
 * returns 1 if it exceeds `threshold`, 0 if not, a negative code on error.
 * b_l in {1, 2, 4, 8, GACT_BITS_UNCOMPRESSED}: a tensor that
 * gact_allocate_bits_levels left uncompressed counts with S(32) = (2^32-1)^-2.
 */
int gact_variance_alert(const float *h_sensitivity, const int32_t *h_bits, int L,
                        double grad_var, double threshold, double *h_ratio);

/*
 * Bit allocator (host only, synchronous; Eq. (ilp), Sec. 4.1-4.2).
 *   h_sensitivity in  c_l >= 0, finite, L floats (Alg. 1's estimate)
 *   h_numel       in  D_l >= 0, L values
 *   avg_bit_budget    budget = floor(avg * sum_l D_l) bits; must be >= 1
 *   h_bits_out    out b_l in {1,2,4,8}
 * Greedy descent from 8 bits: repeatedly apply the one-level step
 * (8->4, 4->2, 2->1 of one tensor) with the least added variance per bit
 * saved, c_l (S(lo) - S(hi)) / (D_l (hi - lo)) in binary64, ties to the lowest
 * index, until sum b_l D_l <= budget.  Tensors with D_l = 0 keep 8.
 */
int gact_allocate_bits(const float *h_sensitivity, const int64_t *h_numel, int L,
                       double avg_bit_budget, int32_t *h_bits_out);

/*
 * The same program over a caller-given level set: h_levels is strictly
 * ascending and drawn from {1, 2, 4, 8, GACT_BITS_UNCOMPRESSED}; the descent
 * starts from the top level and avg_bit_budget must be >= the lowest.  With 32
 * in the set the most sensitive tensors can stay uncompressed, as in the
 * paper's experiments (Sec. 6.1), S(32) = (2^32-1)^-2.
 * gact_allocate_bits is this call with levels {1, 2, 4, 8}.
 */
int gact_allocate_bits_levels(const float *h_sensitivity, const int64_t *h_numel, int L,
                              double avg_bit_budget, const int32_t *h_levels, int n_levels,
                              int32_t *h_bits_out);

#ifdef __cplusplus
}
#endif
#endif /* GACT_H */
