/*
 * rtopk.h -- C ABI of the MI355X (gfx950) rTop-k hot path.
 *
 * Two operations, both taken from the paper's problem statement (Section III,
 * Algorithm 1): per worker, sparsify the error-compensated gradient with the
 * rTop-k operator of Definition 3; on the master, average the n sparse
 * messages into one dense update.
 *
 * Conventions for every entry point
 *   - Pointers marked "device" are HIP device pointers valid on the current
 *     device; pointers marked "host" are ordinary host pointers.
 *   - The library allocates no device memory and never synchronises the host
 *     (rtopk_encode_stats excepted). All state that links one call to the
 *     next is in the caller's buffers (the residual) and arguments (step); the
 *     library itself only remembers, per device, the launch width of its
 *     streaming kernel. Work is enqueued on `stream` (a hipStream_t, may be
 *     NULL for the default stream) and the call returns at once. The caller
 *     owns all buffers, workspace included, and must keep them alive until the
 *     stream has drained.
 *   - The hot-path calls only launch kernels (what must start at zero is
 *     cleared by those kernels, not by memset nodes): they may be issued on a
 *     stream that is being captured into a HIP graph and replayed. A replay
 *     repeats the arguments it was captured with, the step number included:
 *     rtopk_encode and rtopk_encode_batch in a graph draw the SAME random
 *     subset on every replay, which under error feedback starves the members
 *     with large keys. A loop that replays a graph uses
 *     rtopk_encode_batch_device_step, which reads the step number from device
 *     memory that the graph itself advances.
 *   - Diagnostics (statistics of the last encode, event tracing, hooks that
 *     force the exact fallback paths, a streaming calibration kernel) are not
 *     part of this interface: they are declared in rtopk_diag.h.
 *   - Two calls may run concurrently only with distinct workspaces, residuals
 *     and outputs.
 *   - Return value: RTOPK_OK or a negative error code; rtopk_strerror() gives
 *     a static description. Argument checks are made on the host before
 *     anything is launched; a failed check launches nothing.
 *   - Results are a pure function of the argument values and buffer contents:
 *     they do not depend on grid size, stream or run, nor on what the
 *     workspace held. Against another
 *     implementation of the same arithmetic they agree bit for bit, with one
 *     exception IEEE 754 leaves open: when an addition meets two not-a-number
 *     operands with different payloads (two workers sending NaN for one
 *     coordinate; a NaN gradient entry on a NaN residual entry), the result is
 *     a NaN whose payload is the hardware's choice.
 */
#ifndef RTOPK_H
#define RTOPK_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define RTOPK_OK 0
#define RTOPK_EINVAL (-1)     /* null pointer, or sizes outside 1 <= k <= r <= d < 2^32, n < 1, aliasing */
#define RTOPK_EWORKSPACE (-2) /* workspace null, misaligned (256 bytes) or too small */
#define RTOPK_EHIP (-3)       /* a HIP call or kernel launch failed */
#define RTOPK_ETOOLARGE (-4)  /* sizes beyond the built-in scratch of rtopk_aggregate_update_static */

/* Bytes of device workspace one rtopk_encode call needs for these sizes: the
 * caller-owned scratch memory behind Algorithm 1's node-side step (nothing of
 * it survives the call). bytes: host pointer, written on success. */
int rtopk_encode_workspace_bytes(uint64_t d, uint64_t r, uint64_t k, uint64_t *bytes);

/* Bytes of device workspace rtopk_aggregate (Algorithm 1's master step) needs
 * for these sizes; currently 0, the argument is kept for the interface. */
int rtopk_aggregate_workspace_bytes(uint64_t d, uint32_t n, uint64_t k, uint64_t *bytes);

/*
 * One node-side step of Algorithm 1 for one worker:
 *     a <- grad + residual            (error compensation, one binary32 add)
 *     U <- rTop-k selection on a      (Definition 3: a uniformly random
 *                                      k-subset of the r largest-magnitude
 *                                      coordinates, Definition 1)
 *     message <- {(i, a_i) : i in U}
 *     residual <- a - message         (a_i where not sent; a_i - a_i where sent)
 *
 * Choices the paper leaves open, fixed here so the result is unique:
 *   magnitude order = order of the low 31 bits of the binary32 pattern; equal
 *   magnitudes: lower index first; U = the k members of the top-r set with
 *   the smallest (K(i), i), K(i) = first two output words (word0 << 32 |
 *   word1) of Philox4x32-10 with counter (i, 0, step_lo, step_hi) and key
 *   (seed_lo, seed_hi).
 *
 * grad       device, [d] binary32, read only
 * residual   device, [d] binary32, in: m_t, out: m_{t+1}; must not overlap grad
 * d, r, k    1 <= k <= r <= d < 2^32. r == k is the top-k operator (no key is
 *            ever computed), r == d the random-k operator (no magnitude is
 *            ever compared: no estimate, no histogram, no threshold)
 * seed,step  select the random subset; a fresh `step` gives a fresh subset,
 *            distinct `seed`s give independent workers
 * out_idx    device, [k] uint32, the set U in strictly ascending order
 * out_val    device, [k] binary32, out_val[j] = a[out_idx[j]]
 * workspace  device, 256-byte aligned, >= rtopk_encode_workspace_bytes(d,r,k):
 *            one byte per element (every chunk of the vector owns room for an
 *            eighth of its elements as 8-byte candidates; a chunk that keeps
 *            more is read from the residual buffer itself) plus about 10 MB
 *            of histograms, lists and counters; contents on entry are
 *            irrelevant, contents on return unspecified but for its first
 *            32-bit word: once the call's kernels have run it holds the
 *            call's error flags, 0 when the message is valid, non-zero when
 *            an internal consistency check failed (a selection found no
 *            element of its rank, the winners did not add up to k, a bounded
 *            wait inside a kernel ran out) and the outputs must be discarded.
 *            A caller that wants to know without stopping the stream copies
 *            that word asynchronously; no input in the domain above is known
 *            to set it
 * stream     hipStream_t
 */
int rtopk_encode(const float *grad, float *residual,
                 uint64_t d, uint64_t r, uint64_t k,
                 uint64_t seed, uint64_t step,
                 uint32_t *out_idx, float *out_val,
                 void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * The same step of Algorithm 1 for n independent vectors of equal sizes in
 * one call: the n workers that Algorithm 1's node loop runs over (when one
 * device holds several of them), or the tensors of one model. Member i is
 * computed exactly as rtopk_encode(grad[i], residual[i], d, r, k, seed[i],
 * step, out_idx[i], out_val[i], ...) computes it, bit for bit; the members
 * only share kernel launches (up to 16 per launch), so the short kernels of
 * all members run side by side and the streaming kernel does not drain in
 * between.
 *
 * grad, residual, out_idx, out_val   HOST arrays of n device pointers each,
 *            read during the call; every pointer as for rtopk_encode. No two
 *            members may share or overlap a residual or an output buffer.
 * seed       HOST array of n seeds
 * workspace  device, 256-byte aligned, >= n * rtopk_encode_workspace_bytes(d,r,k);
 *            member i uses the i-th slice of that size (its first word holds
 *            member i's error flags), and rtopk_encode_stats on the slice's
 *            address reports on member i
 */
int rtopk_encode_batch(uint32_t n,
                       const float *const *grad, float *const *residual,
                       uint64_t d, uint64_t r, uint64_t k,
                       const uint64_t *seed, uint64_t step,
                       uint32_t *const *out_idx, float *const *out_val,
                       void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * rtopk_encode_batch with the step number of Algorithm 1's loop read from
 * device memory when the kernels run, not passed by value when they are
 * enqueued: for a step captured once into a HIP graph and replayed every
 * iteration, with a small kernel in the same graph (or any other work on the
 * stream) advancing *step_device in between. Every replay then draws a fresh
 * uniform subset (Definition 3), as a loop of rtopk_encode_batch calls with
 * step = 0, 1, 2, ... does; the results are the same bit for bit.
 *
 * step_device   device, one uint64, 8-byte aligned; read by every kernel of
 *               the call, so it must not change while the call's kernels run
 * everything else as for rtopk_encode_batch (n = 1 serves a single vector)
 */
int rtopk_encode_batch_device_step(uint32_t n,
                                   const float *const *grad, float *const *residual,
                                   uint64_t d, uint64_t r, uint64_t k,
                                   const uint64_t *seed, const uint64_t *step_device,
                                   uint32_t *const *out_idx, float *const *out_val,
                                   void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * Master step of Algorithm 1: out = (1/n) * sum_{w<n} message_w as a dense
 * vector. Every coordinate is divided by n, whether or not all workers sent
 * it; coordinates nobody sent are +0. Sums are formed in binary32 starting
 * from +0, adding workers in the order 0..n-1 (entries of one message in
 * position order, so a repeated index is simply added again), followed by
 * one correctly rounded binary32 division by (float)n. No floating-point
 * atomics are used, so the result is reproducible bit for bit.
 *
 * idx   device, [n*k] uint32, worker-major: worker w owns [w*k, (w+1)*k);
 *       each worker's slice must be sorted ascending (as rtopk_encode emits
 *       it); every index must be < d (precondition, not checked)
 * val   device, [n*k] binary32
 * out   device, [d] binary32, fully overwritten
 * workspace  device, 256-byte aligned, >= rtopk_aggregate_workspace_bytes
 */
int rtopk_aggregate(const uint32_t *idx, const float *val,
                    uint32_t n, uint64_t k, uint64_t d,
                    float *out,
                    void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * Both master lines of Algorithm 1 in one step, without the dense average in
 * between: omega[i] <- omega[i] - eta * scale * (1/n) * sum_{w<n} message_w[i].
 * scale = 1 is the algorithm as printed. scale = r/k divides what a node kept
 * by the fraction k/r it kept of its top-r set, in the manner of the
 * estimator in the proof of the estimation upper bound, which divides the
 * subsampled vector by its subsampling fraction; the mean over the random
 * subsets then equals the top-r part of the node's vector.
 *
 * Arithmetic, all binary32: the sum and the division by n exactly as in
 * rtopk_aggregate; the step c = eta * scale rounded once; then one fused
 * multiply-add, omega[i] = fma(-c, average[i], omega[i]). A coordinate whose
 * average is zero (nobody sent it, what was sent cancels, or the quotient by
 * n underflows) is not written and keeps its bits; for finite c and omega[i]
 * that is the number the formula gives, up to the sign of a zero weight.
 * Reproducible bit for bit; no atomics.
 *
 * idx, val, n, k, d   as for rtopk_aggregate; n <= 65535
 * omega   device, [d] binary32, updated in place. Only weights that move are
 *         written; where many indices fall close together, the 16-byte groups
 *         around them are read and written back whole, the unmoved weights
 *         with the bits they had. Must not overlap idx, val or workspace.
 * workspace  device, 256-byte aligned, >= rtopk_aggregate_update_workspace_bytes
 *            (4 bytes per worker and per 2048 coordinates); contents on entry
 *            are irrelevant, contents on return unspecified
 * Errors: RTOPK_EINVAL, RTOPK_EWORKSPACE, RTOPK_EHIP as for rtopk_encode.
 */
int rtopk_aggregate_update_workspace_bytes(uint64_t d, uint32_t n, uint64_t k, uint64_t *bytes);
int rtopk_aggregate_update(const uint32_t *idx, const float *val,
                           uint32_t n, uint64_t k, uint64_t d,
                           float eta, float scale,
                           float *omega,
                           void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * rtopk_aggregate_update for callers that cannot allocate device memory and
 * have no workspace to pass: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc. Same arguments, same kernels and
 * the same results bit for bit as rtopk_aggregate_update, but the table of
 * tile starts lives in a device array of RTOPK_STATIC_SCRATCH_BYTES that is
 * part of the library (every GPU the library runs on holds it until the
 * process ends). The call allocates nothing and calls no allocating routine.
 *
 * Limit: (ceil(d / 2048) + 1) * n * 4 bytes, rounded up to 256, must not
 * exceed RTOPK_STATIC_SCRATCH_BYTES (16 MiB: d = 2^28 with up to 31 workers,
 * d = 2^32 - 1 with one); beyond it the call returns RTOPK_ETOOLARGE and
 * launches nothing.
 * The first call on a device looks up the array's address (it may load the
 * library's device code): make it once outside any stream capture.
 * All calls on one GPU share the one array: two calls whose kernels may
 * overlap (different streams, no ordering between them) race; calls on one
 * stream, or ordered by events, are safe. Nothing in the array has to be
 * cleared between calls: every word a call reads it has written itself.
 */
#define RTOPK_STATIC_SCRATCH_BYTES (16u << 20)
int rtopk_aggregate_update_static(const uint32_t *idx, const float *val,
                                  uint32_t n, uint64_t k, uint64_t d,
                                  float eta, float scale,
                                  float *omega, void *stream);

/*
 * The master's update with momentum, the optimiser the experiments section
 * uses (momentum SGD; the paper prints no formula, this is the common one):
 *     ghat = (1/n) * sum_{w<n} message_w
 *     velocity[i] <- mu * velocity[i] + scale * ghat[i]
 *     omega[i]    <- omega[i] - eta * velocity[i]
 * for every i: the velocity decays where nothing was sent, so this is a dense
 * pass over both arrays (16 bytes per coordinate plus the messages). mu = 0
 * moves the weights as rtopk_aggregate_update does.
 *
 * Arithmetic, all binary32: the average exactly as in rtopk_aggregate;
 * u = scale * average (one rounding); velocity = fma(mu, velocity, u);
 * omega = fma(-eta, velocity, omega) with the rounded new velocity.
 * Reproducible bit for bit; no atomics, no workspace.
 *
 * idx, val, n, k, d   as for rtopk_aggregate
 * omega, velocity     device, [d] binary32 each, updated in place; they must
 *                     not overlap each other, idx or val
 */
int rtopk_aggregate_update_momentum(const uint32_t *idx, const float *val,
                                    uint32_t n, uint64_t k, uint64_t d,
                                    float eta, float scale, float mu,
                                    float *omega, float *velocity, void *stream);

/*
 * ---------------------------------------------------------------------------
 * Matrix parameters: what stands before and after the sparse exchange in a
 * training step. A layer's products in 8-bit integers give its outputs and the
 * binary32 gradient that rtopk_encode takes; the master's step below moves a
 * matrix by its orthogonalised momentum. Matrices are row-major, `ld` is the
 * distance of their rows in elements.
 * ---------------------------------------------------------------------------
 */
#define RTOPK_F32 0
#define RTOPK_BF16 1
#define RTOPK_F16 2

#define RTOPK_ROWS 0
#define RTOPK_COLUMNS 1

/*
 * Quantisation to 8 bits with a scale for each row (a token, an output
 * channel) or for each column:
 *     scale = max |x| / 127,  q = round to nearest, ties to even (x / scale)
 * both divisions binary32. Along RTOPK_ROWS, q is [rows][ldq] as x is, scale
 * [rows]. Along RTOPK_COLUMNS the matrix is also turned over, q is [cols][ldq]
 * with the rows of x along its rows, scale [cols]: the contraction of a
 * gradient runs over the tokens, and the product below over rows.
 * A row (column) whose scale would be below 2^-126 gets scale 0 and numbers 0;
 * one that holds an infinity or a not-a-number gets scale NaN and numbers 0,
 * so that everything it goes into is NaN.
 *
 * x      device, [rows][ldx] of `type`; any alignment of its elements' size,
 *        16-byte aligned rows are read fastest
 * rows   0 .. 2^22 (0: nothing to do along rows, scales 0 along columns)
 * cols   1 .. 2^22; cols <= ldx <= 2^22
 * q      device; what lies between the numbers and ldq is not written. Rows
 *        that start on 16 bytes (base and ldq) let the product load them
 *        directly
 * workspace  device, 256-byte aligned, >= rtopk_quantize_i8_workspace_bytes
 *        (0 along rows)
 */
int rtopk_quantize_i8_workspace_bytes(uint64_t rows, uint64_t cols, int along, uint64_t *bytes);
int rtopk_quantize_i8(const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ldx,
                      int along, int8_t *q, uint64_t ldq, float *scale,
                      void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * out[i][j] = a_scale[i] * b_scale[j] * sum_k a[i][k] * b[j][k] + bias[j].
 * The sums are exact (any of -128 .. 127); they are rounded to binary32 once,
 * then take the scales and the bias in binary32, and the type of `out`.
 *
 * a      device, [m][lda] int8; a_scale device, [m]
 * b      device, [n][ldb] int8; b_scale device, [n]
 * bias   device, [n] binary32, or null
 * m, n, k  0 .. 2^22 (k = 0: out is the bias), lda, ldb <= 2^22
 * out    device, [m][ldo] of out_type; must not overlap an input
 * workspace  device, 256-byte aligned, >= rtopk_matmul_i8_workspace_bytes
 */
int rtopk_matmul_i8_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, uint64_t *bytes);
int rtopk_matmul_i8(const int8_t *a, const float *a_scale, const int8_t *b, const float *b_scale,
                    const float *bias, uint64_t m, uint64_t n, uint64_t k,
                    uint64_t lda, uint64_t ldb, void *out, int out_type, uint64_t ldo,
                    void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * A layer's forward product: x quantised by row (token) as rtopk_quantize_i8
 * does, times weights that are quantised already: out = x w^T + bias.
 *
 * x      device, [m][ldx] of `type`, m tokens (0 .. 2^22) of k numbers
 * w      device, [n][ldw] int8, a row for each output channel; w_scale [n]
 * the rest as above; both calls' sizes limit as rtopk_matmul_i8's do, k and n
 * are at least 1
 */
int rtopk_linear_i8_workspace_bytes(uint64_t m, uint64_t k, uint64_t n, uint64_t *bytes);
int rtopk_linear_i8(const void *x, int type, uint64_t m, uint64_t k, uint64_t ldx,
                    const int8_t *w, const float *w_scale, uint64_t n, uint64_t ldw,
                    const float *bias, void *out, int out_type, uint64_t ldo,
                    void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * Its backward products, the gradients passed straight through the rounding:
 *     dx = dy w        dy quantised by row, w by column
 *     dw = dy^T x      both quantised by column (over the tokens)
 *     db = sum of dy's rows, in binary32 or more
 *
 * dy, x  device, [m][lddy] and [m][ldx] of `type`
 * w_turned, w_turned_scale  device, [k][ldw] int8 and [k]: the weights [n][k]
 *        quantised along RTOPK_COLUMNS
 * dx     device, [m][lddx] of `type`, or null
 * dw     device, [n][lddw] binary32, or null (then x is not read): with
 *        lddw = k the gradient as rtopk_encode takes it
 * db     device, [n] binary32, or null; only with dw
 * m = 0 writes zeros to dw and db
 */
int rtopk_linear_i8_backward_workspace_bytes(uint64_t m, uint64_t k, uint64_t n, uint64_t *bytes);
int rtopk_linear_i8_backward(const void *dy, const void *x, int type,
                             uint64_t m, uint64_t k, uint64_t n, uint64_t lddy, uint64_t ldx,
                             const int8_t *w_turned, const float *w_turned_scale, uint64_t ldw,
                             void *dx, uint64_t lddx, float *dw, uint64_t lddw, float *db,
                             void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * Orthogonalises `count` matrices of equal shape: with X = G / (|G|_F + eps),
 * turned over if G has more rows than columns, each step takes its three
 * coefficients (a, b, c) and
 *     A = X X^T,  X <- a X + (b A + c A A) X
 * which moves every singular value s of X to a s + b s^3 + c s^5 and leaves
 * the singular vectors. (3.4445, -4.7750, 2.0315) five times is in common use
 * for updates of neural networks. Members are independent of each other, up to
 * 16 share launches.
 *
 * products  RTOPK_PRODUCTS_PAIRS: numbers between the products are pairs of
 *        halves (22 bits), each product is three half products: about as exact
 *        as binary32 (relative error of the result 10^-6 to 10^-5 for a
 *        gradient, and 10^-7 s where one direction is s > 100 times as strong
 *        in each element as the others; binary32 the same).
 *        RTOPK_PRODUCTS_HALVES: halves (11 bits, three more than bfloat16
 *        has), down to a third of the time: 2048 times those errors, 8 10^-4
 *        for noise. A bfloat16 x with a direction of s = 30, 100, 1000 comes
 *        out with 1.5 10^-3, 5 10^-3 and 2 10^-2 (a bfloat16 result's own
 *        rounding is 1.7 10^-3), a binary32 x with 6 10^-3, 2 10^-2 and 0.12:
 *        for matrices that are known to have no such direction
 * x      HOST array of device pointers to [rows][ldx] of `type`
 * out    HOST array of device pointers to [rows][ldo] of out_type; may be x
 * rows, cols  1 .. 2^21, rows * cols < 2^32
 * coefficients  HOST, [steps][3], 1 <= steps <= 64, read during the call. If
 *        singular values s that start in [0, 1] can pass 7.5 (or a + b s^2 +
 *        c s^4 can pass 30), the call returns RTOPK_EINVAL
 * eps    >= 0. A matrix of zeros gives zeros (eps = 0 too); one that holds an
 *        infinity or a not-a-number gives NaN everywhere. |G|_F may be far below
 *        eps: down to 2^-100 eps the result keeps its bits where a is not
 *        much smaller than |b| and |c| (A is computed to 2^-22, or 2^-11, of
 *        what its diagonal would be without eps)
 * workspace  device, 256-byte aligned, >= rtopk_orthogonalize_workspace_bytes
 */
#define RTOPK_PRODUCTS_PAIRS 0
#define RTOPK_PRODUCTS_HALVES 1
int rtopk_orthogonalize_workspace_bytes(uint32_t count, uint64_t rows, uint64_t cols, int products,
                                        uint64_t *bytes);
int rtopk_orthogonalize(uint32_t count, const void *const *x, int type,
                        uint64_t rows, uint64_t cols, uint64_t ldx,
                        uint32_t steps, const float *coefficients, float eps, int products,
                        void *const *out, int out_type, uint64_t ldo,
                        void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * The master's step for `count` matrix parameters of equal shape, each with
 * messages of its own from n workers, indices counted along the flat matrix:
 *     average  = (1/n) sum of the messages, as rtopk_aggregate forms it
 *     u        = scale * average
 *     velocity = mu * velocity + u
 *     G        = mu * velocity + u (nesterov != 0), or velocity
 *     omega    = (1 - eta * decay) * omega - eta * gain * orthogonalised(G)
 * u rounded, the next two fused multiply-adds; keep = 1 - eta * decay and
 * step = eta * gain rounded to binary32, omega = fma(-step, O, keep * omega).
 *
 * idx, val         HOST arrays of device pointers, each [n*k] as for
 *                  rtopk_aggregate with d = rows * cols
 * omega, velocity  HOST arrays of device pointers, [rows * cols] binary32,
 *                  updated in place; no two of them may overlap
 * the rest as for rtopk_orthogonalize
 */
int rtopk_aggregate_update_orthogonal_workspace_bytes(uint32_t count, uint64_t rows, uint64_t cols,
                                                      int products, uint64_t *bytes);
int rtopk_aggregate_update_orthogonal(uint32_t count, const uint32_t *const *idx,
                                      const float *const *val, uint32_t n, uint64_t k,
                                      uint64_t rows, uint64_t cols, float eta, float scale,
                                      float mu, int nesterov, float decay, float gain,
                                      uint32_t steps, const float *coefficients, float eps,
                                      int products, float *const *omega, float *const *velocity,
                                      void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * The same products in 4-bit floating point with a scale for each block of 32
 * numbers of the contraction. A number is one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and
 * their negatives (sign, two exponent bits, one mantissa bit: E2M1), two a
 * byte, the even one in the lower half; a scale is the byte b for 2^(b - 127),
 * 255 for NaN. A quantised matrix is q, [rows][ldq] BYTES with (k + 1) / 2 of
 * them in a row (the last half byte of an odd k is 0), and scale, turned over:
 * [blocks][lds] bytes, a row of the matrix's `rows` scales for each of
 * the (k + 31) / 32 blocks.
 *
 * rtopk_quantize_mx4 takes for each block, with RTOPK_NEAREST, the least scale
 * with max |x| < 7 scale, and rounds x / scale to the nearest number, ties to
 * even: no number is off by more than half the step of numbers around it. With
 * RTOPK_DRAWN, the least scale with max |x| <= 6 scale, and x / scale goes to
 * one of the two numbers around it by chance: up where a 16-bit draw u has
 * u + 1/2 < 65536 f, f being how far it is from the lower one to the upper one
 * in magnitude. The mean is x to within 2^-17 of a step, as a gradient needs
 * it. The least scale of all is 2^-127. A block that holds an infinity or a
 * not-a-number gets scale NaN and numbers 0, so that everything it goes into is NaN.
 *
 * Draws: number c % 8 of Philox4x32-10's eight 16-bit numbers (word by word,
 * lower half first) for counter (g_lo, what << 24 | g_hi, step_lo, step_hi),
 * key (seed_lo, seed_hi), g = row * 4 * blocks + c / 8 by the row and column c
 * of q, what = 2 along rows, 3 along columns. `step_device`, if not null, is a
 * device uint64 that the step number is read from when the kernels run: a graph that is
 * replayed advances it, and each replay draws afresh. A draw belongs to seed,
 * step and place alone: matrices that are to be drawn independently, as those
 * of two layers in one step, need seeds of their own.
 *
 * x      device, [rows][ldx] of `type`, rows 0 .. 2^22, cols 1 .. 2^22 <= ldx <= 2^22
 * along  RTOPK_ROWS: q [rows][ldq], scale [(cols + 31) / 32][lds]; RTOPK_COLUMNS:
 *        turned over, q [cols][ldq] with the rows of x along its rows, scale
 *        [(rows + 31) / 32][lds]. ldq, lds <= 2^22
 * q, scale  device; what lies between a row's end and ldq or lds is not
 *        written. Rows of q that start on 16 bytes (base and ldq) and rows of
 *        scale that start on 4 let the product load them directly
 */
#define RTOPK_NEAREST 0
#define RTOPK_DRAWN 1
int rtopk_quantize_mx4(const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ldx,
                       int along, int rounding, uint64_t seed, uint64_t step, const uint64_t *step_device,
                       uint8_t *q, uint64_t ldq, uint8_t *scale, uint64_t lds, void *stream);

/*
 * Back to numbers: out[r][c] = number * scale in the type of `out` (beyond its
 * largest an infinity). rows, cols  0 .. 2^22: of q's matrix, as it lies
 */
int rtopk_dequantize_mx4(const uint8_t *q, uint64_t rows, uint64_t cols, uint64_t ldq,
                         const uint8_t *scale, uint64_t lds,
                         void *out, int type, uint64_t ldo, void *stream);

/*
 * out[i][j] = sum_k a[i][k] b[j][k] + bias[j], binary32 sums of exact products.
 *
 * a, a_scale  device, a quantised matrix of m rows of k numbers: lda bytes from
 *        row to row, lda_scale from block to block
 * b, b_scale  device, n rows of k numbers
 * bias   device, [n] binary32, or null
 * m, n, k  0 .. 2^22 (k = 0: out is the bias); all distances of operands <= 2^22
 * out    device, [m][ldo] of out_type; must not overlap an input
 * workspace  device, 256-byte aligned, >= rtopk_matmul_mx4_workspace_bytes
 */
int rtopk_matmul_mx4_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, uint64_t *bytes);
int rtopk_matmul_mx4(const uint8_t *a, const uint8_t *a_scale, const uint8_t *b, const uint8_t *b_scale,
                     const float *bias, uint64_t m, uint64_t n, uint64_t k,
                     uint64_t lda, uint64_t lda_scale, uint64_t ldb, uint64_t ldb_scale,
                     void *out, int out_type, uint64_t ldo,
                     void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * A layer's forward product: x, quantised to the nearest along rows on the way,
 * times weights that are quantised already: out = x w^T + bias.
 *
 * x      device, [m][ldx] of `type`, m tokens (0 .. 2^22) of k numbers
 * w, w_scale  device, n rows of k numbers, a row for each output channel
 * the rest as above; k and n are at least 1
 */
int rtopk_linear_mx4_workspace_bytes(uint64_t m, uint64_t k, uint64_t n, uint64_t *bytes);
int rtopk_linear_mx4(const void *x, int type, uint64_t m, uint64_t k, uint64_t ldx,
                     const uint8_t *w, const uint8_t *w_scale, uint64_t n, uint64_t ldw, uint64_t ldw_scale,
                     const float *bias, void *out, int out_type, uint64_t ldo,
                     void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * Its backward products, the gradients passed straight through the rounding:
 *     dx = dy w        dy quantised along rows, w along columns
 *     dw = dy^T x      both quantised along columns (over the tokens)
 *     db = sum of dy's rows, in binary32 or more
 * x is quantised to the nearest, dy by `rounding` with seed and step as in
 * rtopk_quantize_mx4: a seed of its own for each layer.
 *
 * dy, x  device, [m][lddy] and [m][ldx] of `type`
 * w_turned, w_turned_scale  device, k rows of n numbers: the weights [n][k]
 *        quantised along RTOPK_COLUMNS
 * dx     device, [m][lddx] of `type`, or null
 * dw     device, [n][lddw] binary32, or null (then x is not read): with
 *        lddw = k the gradient as rtopk_encode takes it
 * db     device, [n] binary32, or null; only with dw
 * m = 0 writes zeros to dw and db
 */
int rtopk_linear_mx4_backward_workspace_bytes(uint64_t m, uint64_t k, uint64_t n, uint64_t *bytes);
int rtopk_linear_mx4_backward(const void *dy, const void *x, int type,
                              uint64_t m, uint64_t k, uint64_t n, uint64_t lddy, uint64_t ldx,
                              const uint8_t *w_turned, const uint8_t *w_turned_scale,
                              uint64_t ldw, uint64_t ldw_scale,
                              int rounding, uint64_t seed, uint64_t step, const uint64_t *step_device,
                              void *dx, uint64_t lddx, float *dw, uint64_t lddw, float *db,
                              void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * Layer norm over the rows of a matrix, what stands before a layer's product:
 *     mean = sum x / cols,  rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps)
 *     out  = (x - mean) rstd gamma + beta
 * in binary32 (rows of more than 16384 numbers are summed in binary64), off by
 * roundings of x - mean, however far the mean is from zero.
 *
 * x      device, [rows][ldx] of `type`, rows 0 .. 2^22, cols 1 .. 2^22 <= ldx <= 2^22
 * gamma, beta  device, [cols] binary32, or null: 1, 0
 * eps    >= 0. (A row of equal numbers gives beta; with eps = 0 it gives NaN.)
 * out    device, [rows][ldo] of out_type, ldo <= 2^22; may be x itself (types
 *        of one size, ldo = ldx), else must not overlap an input
 * mean, rstd  device, [rows] binary32 each, for the backward pass; or null
 */
int rtopk_layer_norm(const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ldx,
                     const float *gamma, const float *beta, float eps,
                     void *out, int out_type, uint64_t ldo, float *mean, float *rstd, void *stream);

/*
 * Its gradients. With h = (x - mean) rstd and g = dy gamma:
 *     dx     = rstd (g - mean(g) - h mean(g h)) + add
 *     dgamma = sum over rows of dy h,  dbeta = sum over rows of dy
 * The sums over rows are taken in a fixed order: the same bits every time.
 *
 * dy     device, [rows][lddy] of dy_type; x device, [rows][ldx] of `type`
 * mean, rstd  device, [rows], as rtopk_layer_norm leaves them (h is off by what
 *        the mean loses as binary32)
 * gamma  device, [cols], or null: 1
 * add    device, [rows][ldadd] of `type`, or null: the gradient that reaches x
 *        past the norm; only with dx
 * dx     device, [rows][lddx] of `type`, or null; may be dy (types of one size),
 *        x or add itself (equal distances of rows), else must not overlap an input
 * dgamma, dbeta  device, [cols] binary32 each, or null; rows = 0 writes zeros
 * All distances of rows are 2^22 at most.
 * workspace  device, 256-byte aligned, >= rtopk_layer_norm_backward_workspace_bytes;
 *        not read where both dgamma and dbeta are null
 */
int rtopk_layer_norm_backward_workspace_bytes(uint64_t rows, uint64_t cols, uint64_t *bytes);
int rtopk_layer_norm_backward(const void *dy, int dy_type, const void *x, int type, uint64_t rows, uint64_t cols,
                              uint64_t lddy, uint64_t ldx, const float *mean, const float *rstd, const float *gamma,
                              const void *add, uint64_t ldadd, void *dx, uint64_t lddx, float *dgamma, float *dbeta,
                              void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * Dropout, what stands behind a layer's product; the mask is drawn and never
 * stored. With T = p * 65536 rounded to a whole number (ties to even):
 *     out = (u >= T ? x * 65536 / (65536 - T) : 0) + residual
 * in binary32. What is dropped counts as 0, whatever it was. The gradient of x
 * is the same call on out's gradient, with the same p, seed and step and without residual; the
 * residual's is out's gradient itself.
 *
 * Draws: element e = row * cols + col has number e % 8 of the eight 16-bit
 * numbers of counter (g_lo, 1 << 24 | g_hi, step_lo, step_hi), g = e / 8, as
 * above. They do not depend on how the rows lie, and differ from those of
 * rtopk_encode and rtopk_quantize_mx4 with the same seed and step. Two calls
 * with the same seed and step have the same mask, as forward and backward need
 * it; each place of a network needs a seed of its own.
 *
 * x      device, [rows][ldx] of `type`
 * residual  device, [rows][ldr] of out_type, or null
 * out    device, [rows][ldo] of out_type; may be x (types of one size, ldo =
 *        ldx) or residual (ldo = ldr) itself, else must not overlap an input
 * rows, cols  0 .. 2^32 - 1, rows * cols <= 2^40; distances of rows below 2^32
 * p      0 .. 1
 * step_device  a device uint64 that the step number is read from, or null
 */
int rtopk_dropout(const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ldx,
                  const void *residual, uint64_t ldr, void *out, int out_type, uint64_t ldo,
                  double p, uint64_t seed, uint64_t step, const uint64_t *step_device, void *stream);

const char *rtopk_strerror(int code);

/* Library version: major * 10000 + minor * 100 + patch. */
int rtopk_version(void);

#ifdef __cplusplus
}
#endif
#endif /* RTOPK_H */
