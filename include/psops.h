/*
 * psops.h -- C ABI of the B200 PSO-PS parameter-synchronisation library.
 *
 * PSO-PS (Ye, Han, Sun, Lv, "PSO-PS: Parameter Synchronization with Particle
 * Swarm Optimization for Distributed Training of Deep Neural Networks")
 * replaces the averaging step of data-parallel training by a particle-swarm
 * update: the K workers' weight vectors are particles (Table I: position =
 * weights, fitness = training loss), each with a velocity and a personal best,
 * and at every synchronisation point new weights come from Eq. 6 / Eq. 7
 * instead of from the mean.  This library is that synchronisation stage for K
 * particles held as K flat fp32 rows in one GPU's memory.
 *
 * Conventions
 *   - All entry points return 0 (PSOPS_OK) or a negative PSOPS_E* code; none
 *     throws, aborts or prints.  Arguments are validated before any launch.
 *   - "device pointer" = address in the memory of the GPU that was current
 *     when psops_create ran; "host pointer" = ordinary process memory.
 *   - The library allocates no device memory.  The caller owns x, v, pbest,
 *     the workspace, dvec/tvec and the stream, and keeps them alive until
 *     psops_destroy.  The context itself is host memory owned by the library.
 *   - A context belongs to the GPU that was current in psops_create; later
 *     calls switch to that GPU for their duration if another one is current.
 *   - A context is not thread-safe: one host thread at a time per context.
 *     Different contexts are independent (different streams run concurrently).
 *   - Work is enqueued on the stream given at creation.  Calls that fill a
 *     host buffer wait for that stream before they return; the others do not.
 *   - Rows: particle i occupies elements [i*ld, i*ld + N) of x, v and pbest.
 *     Elements [N, ld) of a row are padding and are never written.
 *     If x, v, pbest are 16-byte aligned and ld % 4 == 0 the 128-bit kernels
 *     run; otherwise a scalar variant with identical results runs.
 *   - Random numbers: r1, r2 of Eq. 6 are drawn per (particle, element, sync)
 *     from Philox4x32-10 with counter {element >> 1, particle, sync step, 0}
 *     and key {seed low word, seed high word}; the even element of a pair
 *     takes output words 0,1 and the odd element words 2,3; a word w becomes
 *     (w >> 8) * 2^-24 in [0, 1).  The stream is a pure function of those
 *     indices, so a context has no generator state beyond its step counter.
 */
#ifndef PSOPS_H
#define PSOPS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PSOPS_OK           0
#define PSOPS_EINVAL      -1   /* null pointer, size or hyper-parameter out of range   */
#define PSOPS_EALIGN      -2   /* a device pointer is not 4-byte aligned               */
#define PSOPS_ESTATE      -3   /* call order: e.g. sync before any losses were given   */
#define PSOPS_ENAN        -4   /* a host-supplied loss is NaN                          */
#define PSOPS_EWORKSPACE  -5   /* workspace missing, misaligned (256 B) or too small   */
#define PSOPS_ECUDA       -6   /* a CUDA call failed; psops_last_error has its text    */
#define PSOPS_ENOMEM      -7   /* host allocation of the context failed                */
#define PSOPS_ELIMIT      -8   /* size beyond the built-in scratch (psops_quadratic_fitness_static) */

#define PSOPS_MAX_K     1024

/* psops_config.flags */
#define PSOPS_KEEP_GBEST   1u  /* keep a copy of the gBest row of each sync (+4N bytes of workspace) */
#define PSOPS_QUADRATIC    2u  /* reserve workspace for the on-device quadratic fitness              */
#define PSOPS_GBEST_HISTORY 4u /* gBest = best of all syncs so far instead of this sync's best (+4N bytes) */
#define PSOPS_SEPARATE_SELECT 8u /* always run the selection as a kernel of its own (see psops_sync)       */

/* `which` of psops_get_weights / psops_set_weights */
#define PSOPS_X      0         /* weights  w_i  (position of particle i)     */
#define PSOPS_V      1         /* velocity v_i                               */
#define PSOPS_PBEST  2         /* personal best pBest_i                      */
#define PSOPS_GBEST  3         /* gBest of the last sync (needs KEEP_GBEST)  */

typedef struct psops_ctx psops_ctx;      /* opaque */

/* Hyper-parameters (Table II) and geometry of one swarm. */
typedef struct {
    int32_t  K;              /* particles = workers (Table I) held by this context, 1..PSOPS_MAX_K */
    int32_t  k_first;        /* swarm-wide index of row 0; 0 unless the swarm is sharded    */
    int64_t  N;              /* elements per particle, 1 .. 2^33 - 1                        */
    int64_t  ld;             /* row stride in elements, ld >= N                             */
    float    m_max, m_min;   /* Eq. 5; m_max == m_min gives a constant inertia weight       */
    int64_t  t_max;          /* Eq. 5 denominator (Max_t of Algorithm 1), >= 1              */
    float    c1, c2;         /* acceleration constants of Eq. 6                             */
    uint64_t seed;           /* Philox key                                                  */
    uint32_t flags;          /* PSOPS_KEEP_GBEST | PSOPS_QUADRATIC | PSOPS_GBEST_HISTORY |
                                PSOPS_SEPARATE_SELECT                                       */
    int32_t  K_total;        /* particles in the whole swarm when this context holds a shard
                                [k_first, k_first + K) of it; 0 = not sharded (K_total = K)  */
} psops_config;

/* Bytes of device workspace a context with this configuration needs
 * (0 if the configuration is invalid).  The workspace must be 256-byte
 * aligned. */
size_t psops_workspace_bytes(const psops_config *cfg);

/*
 * Particle initialisation (Algorithm 2): adopt the caller's device rows as the
 * swarm.  d_x, d_v, d_pbest: K rows of stride ld each, fp32, already holding
 * the initial weights, velocities and personal bests (Algorithm 2 clones the
 * weights, so callers normally pass pbest == a copy of x).  pBest_loss starts
 * at +inf (the paper initialises no loss), the sync counter at 0.
 * cuda_stream: a cudaStream_t (NULL = the legacy default stream).
 * Errors: EINVAL, EALIGN, EWORKSPACE, ENOMEM, ECUDA.  On error *out is NULL.
 */
int psops_create(psops_ctx **out, const psops_config *cfg,
                 float *d_x, float *d_v, float *d_pbest,
                 void *d_workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Hand in the current training losses of the whole swarm (the fitness of
 * Table I; lower is better): K floats, K_total on a shard.  on_device == 0: host pointer, checked for NaN (ENAN) and copied
 * before the call returns to the stream (the buffer may be reused at once).
 * on_device != 0: device pointer (4-byte aligned), not inspected and not
 * copied now: the selection kernel of the next psops_sync reads it on the
 * stream (and keeps a copy), so the buffer must stay valid and unchanged until
 * that sync has run.
 */
int psops_set_losses(psops_ctx *ctx, const float *losses, int on_device);

/*
 * One synchronisation: the "t % step == 0" branch of Algorithm 1.
 *   1. gBest = weights of the particle with the smallest loss at this
 *      iteration (Algorithm 3); ties go to the lowest particle index; a NaN
 *      loss never beats a number.
 *   2. every particle with loss_i < pBest_loss_i (strict) sets pBest_i to its
 *      current weights and pBest_loss_i to loss_i.
 *   3. v_i <- m v_i + (c1 r1/lambda)(pBest_i - w_i) + (c2 r2/lambda)(gBest - w_i)
 *      (Eq. 6) and w_i <- w_i + v_i (Eq. 7), with m from Eq. 5 at iteration
 *      t_iter (clamped to t_max).  Rounding sequence per element, all fp32
 *      round-to-nearest: dl = pBest - w; dg = gBest - w; t1 = (c1/lambda) r1;
 *      t2 = (c2/lambda) r2; a0 = m v; v' = fma(t2, dg, fma(t1, dl, a0));
 *      w' = w + v'.
 * If a quadratic fitness is attached (psops_set_quadratic) the losses of the
 * NEW weights are evaluated in the same pass and become the losses of the next
 * sync.  Enqueues work only; the sync counter advances by one.  The counter
 * lives in device memory and is advanced by the selection kernel itself, so a
 * psops_sync recorded into a CUDA graph (with the losses in a device buffer,
 * see psops_set_losses) keeps walking the random stream when the graph is
 * replayed; t_iter and lambda are then the ones given at capture.
 * Launches: a small swarm -- at most 8 particles, no history variant, no fused
 * fitness, and few enough elements that all thread blocks of the update are
 * resident at once (on a B200 about 450,000 with up to 4 particles, 150,000
 * with 5 to 8) -- is launch-bound, and its whole sync is ONE kernel: every
 * thread block recomputes steps 1 and 2 from the K losses, and the block that
 * draws the last ticket of a counter publishes g, the improved mask, pBest_loss
 * and the counter (no block waits for another).  Otherwise, or with
 * PSOPS_SEPARATE_SELECT, a selection kernel runs first and the update kernel
 * behind it.  A swarm of 9 or more particles on few elements (up to 2^19, and
 * few enough that one block column per 1024 elements would leave SMs idle) has
 * its rows split into groups that run side by side; since row g is then read
 * by blocks that do not write it, a small kernel first copies it into the
 * workspace -- up to 32 particles that kernel also does the selection (two
 * launches per sync), beyond 32 or with PSOPS_SEPARATE_SELECT the selection
 * kernel runs in front of it (three).  The results are identical bit for bit in
 * every form.
 * Cache policy: of the arrays x, v, pbest (4 K N bytes each) as many as fit
 * together in about half of the GPU's L2 cache are accessed with ordinary
 * loads and stores, so that the next sync finds them there; the others, and
 * everything in a swarm far larger than L2, are streamed (evict-first).
 * Errors: EINVAL (t_iter < 0, lambda < 1 or not finite), ESTATE (no losses
 * yet), ECUDA.
 */
int psops_sync(psops_ctx *ctx, int64_t t_iter, float lambda);

/*
 * Same synchronisation for callers whose weights live in host memory (the
 * workers' side of Algorithm 1: gather weights and losses, distribute new
 * weights).  h_x_in: K rows of stride h_in_ld (>= N) with the workers' current
 * weights; h_losses: K losses; h_x_out: K rows of stride h_out_ld receiving
 * the new weights (may equal h_x_in).  Velocities and personal bests stay on
 * the device.  Copies and kernels are pipelined over element ranges; the call
 * returns when h_x_out is complete.  Pinned host memory gives full speed.
 * Errors: as psops_sync, plus ENAN.  Also on an error from the CUDA runtime the
 * call returns only after every copy and kernel it had queued has finished, so
 * the host buffers may be freed at once; the swarm's state is then undefined
 * (some element ranges updated, others not).
 */
int psops_sync_host(psops_ctx *ctx, const float *h_x_in, int64_t h_in_ld,
                    const float *h_losses, int64_t t_iter, float lambda,
                    float *h_x_out, int64_t h_out_ld);

/*
 * Page-lock (pin) a host buffer that psops_sync_host will use, and release it
 * again.  With ordinary pageable memory the copies of psops_sync_host are
 * staged by the driver and run several times slower (measured: 6x); pin the
 * buffers once, reuse them for every sync, unregister before freeing them.
 * Registering an already registered range is not an error.  EINVAL, ECUDA.
 */
int psops_host_register(void *host_ptr, size_t bytes);
int psops_host_unregister(void *host_ptr);

/*
 * Particle-sharded synchronisation: each GPU holds K of the swarm's K_total
 * particles (psops_config.k_first / K_total) and only the best particle's
 * weights travel -- the exchange Algorithm 3 describes as a gather of all
 * particles reduces to an all-gather of K_total losses plus one broadcast of N
 * floats.  Per sync, on every shard:
 *   1. psops_set_losses with all K_total losses (the caller's all-gather);
 *   2. psops_shard_select: Algorithm 3 and the pBest branch over the whole
 *      swarm; *g receives the swarm-wide gBest index (waits for the stream);
 *   3. the shard that holds particle g copies that row out (psops_get_weights)
 *      and the caller broadcasts it into a buffer in every GPU's own memory;
 *   4. psops_shard_update: Eq. 6 / Eq. 7 for this shard's particles with gBest
 *      read from d_gbest_row (N floats, device pointer, 16-byte aligned on the
 *      128-bit path).  Random draws use the swarm-wide particle index, so the
 *      result is that of one unsharded psops_sync.  The shard that holds
 *      particle g may pass that row of its own x directly: every element of
 *      gBest is read by the thread that later overwrites it.
 *      psops_shard_update_range does step 4 for elements [first_elem,
 *      last_elem) only, so that the broadcast can travel in pieces and the
 *      update of one piece runs while the next is still on the wire: call it
 *      with consecutive ranges from 0 to N (first_elem a multiple of 4,
 *      last_elem a multiple of 4 or N; d_gbest_row always points at element 0 of
 *      the row, of which only the range is read); the sync counter advances when
 *      the range that ends at N has been enqueued.
 * psops_shard_select waits only for the selection kernel (an event behind it;
 * g arrives through a page-locked word the kernel writes), not for later work.
 * psops_sync, psops_sync_host, psops_average and psops_ssgd return ESTATE on a
 * sharded context (they need the whole swarm).  The quadratic fitness and
 * PSOPS_GBEST_HISTORY are not available on shards; PSOPS_KEEP_GBEST is (the
 * shard keeps a copy of the row it was given).
 * Errors: EINVAL, EALIGN, ESTATE (no losses / update without select / a second
 * select before the update is complete / a range out of order), ECUDA.
 */
int psops_shard_select(psops_ctx *ctx, int *g);
int psops_shard_update(psops_ctx *ctx, int64_t t_iter, float lambda, const float *d_gbest_row);
int psops_shard_update_range(psops_ctx *ctx, int64_t t_iter, float lambda, const float *d_gbest_row,
                             int64_t first_elem, int64_t last_elem);

/*
 * gBest from the history of all particles (the standard-PSO framework of
 * Section II-C, step 3, in place of Algorithm 3's best-of-this-iteration):
 * with PSOPS_GBEST_HISTORY the context remembers the best row ever selected
 * and its loss; a sync's arg-min particle replaces it only on a strictly
 * smaller loss (or when nothing is remembered yet), and Eq. 6 uses the
 * remembered row.  psops_get_weights(PSOPS_GBEST) returns that row.  These two
 * calls move the remembered loss (and, for set, the row) for checkpoint/resume.
 */
int psops_get_history(psops_ctx *ctx, float *gbest_loss, int *valid);
int psops_set_history(psops_ctx *ctx, float gbest_loss, const float *gbest_row, int row_on_device);

/*
 * Synchronous SGD as the paper states it beside parameter averaging
 * (Section II-B): w <- w + (alpha / K) sum_k grad_k, written to every row of x
 * (the new weight is computed from row 0).  d_grad: K rows of stride grad_ld
 * (>= N), device pointer.  fp32: gradients summed in worker order, one division
 * alpha / K, one product, one addition.  v, pbest and the sync counter are
 * untouched.
 */
int psops_ssgd(psops_ctx *ctx, const float *d_grad, int64_t grad_ld, float alpha);

/*
 * Parameter averaging, the baseline the paper compares with (Section II-B,
 * step 5): every w_i <- (1/K) sum_k w_k.  fp32 sum in particle order, one
 * division.  Velocities, personal bests and the sync counter are untouched.
 */
int psops_average(psops_ctx *ctx);

/*
 * Copy one row out.  which = PSOPS_X / PSOPS_V / PSOPS_PBEST with particle k in
 * [0, K), or PSOPS_GBEST (k ignored): the gBest row used by the last sync,
 * available only with PSOPS_KEEP_GBEST (else ESTATE, as the pre-update row no
 * longer exists).  dst receives N floats; dst_on_device selects the kind of
 * pointer; a host destination is complete on return.
 */
int psops_get_weights(psops_ctx *ctx, int which, int k, float *dst, int dst_on_device);

/* Overwrite row k of x, v or pbest with N floats from src (host or device). */
int psops_set_weights(psops_ctx *ctx, int which, int k, const float *src, int src_on_device);

/*
 * Selection results of the last sync, copied to host memory (each pointer may
 * be NULL): *g = gBest index; improved_words[(K+31)/32], bit i set when
 * particle i improved; pbest_loss[K] after the update.  Waits for the stream.
 * ESTATE before the first sync.
 */
int psops_sync_info(psops_ctx *ctx, int *g, uint32_t *improved_words, float *pbest_loss);

/* The K losses currently held on the device, to dst (host or device). */
int psops_get_losses(psops_ctx *ctx, float *dst, int dst_on_device);

/*
 * Attach the quadratic stand-in fitness f(w) = sum_j dvec_j (w_j - tvec_j)^2
 * (device pointers, N floats each, borrowed; both NULL detaches).  Needs
 * PSOPS_QUADRATIC.  The summation order is fixed so that results are
 * reproducible bit for bit: fp32 terms dvec*(e*e) widened to fp64; four
 * consecutive terms added left to right; 32 such sums (128 elements) combined
 * by the butterfly a[l] += a[l ^ off], off = 16..1; tile sums added into 1024
 * slots (tile m -> slot m % 1024, increasing m, from +0.0); slots combined as
 * 32 butterflies of 32 and the 32 results added in order; rounded to fp32.
 */
int psops_set_quadratic(psops_ctx *ctx, const float *d_dvec, const float *d_tvec);

/* losses <- f(current weights) for every particle (the evaluation that
 * precedes the first sync). */
int psops_eval_quadratic(psops_ctx *ctx);

/*
 * (No counterpart in the paper: an addition for callers that cannot allocate.)
 * The quadratic fitness of K rows without any workspace and without a context:
 * d_loss[i] = f(row i of d_x), the same value, bit for bit, that
 * psops_eval_quadratic produces.  It is meant for code that has no way to get
 * device memory when it needs the value: inside a loop whose framework already
 * owns all of the GPU's memory through its caching allocator, in a plug-in that
 * is handed nothing but input and output buffers, or where cudaMalloc/cudaFree
 * are off limits because they stall every stream of the device.  The call
 * itself allocates nothing, on the host or on the device.
 *   d_x            K rows of stride ld (>= N) fp32, device pointer
 *   d_dvec, d_tvec N fp32 each, device pointers
 *   d_loss         K fp32, device pointer, written on the stream
 *   cuda_stream    a cudaStream_t (NULL = legacy default stream); work is only
 *                  enqueued
 * The intermediate tile sums go to an array of PSOPS_STATIC_SCRATCH_DOUBLES
 * doubles (8 MiB) that is built into the library and therefore occupies that
 * much memory on every GPU that loads it until the process exits.  A problem
 * with K * ceil(N/128) above that number is refused with PSOPS_ELIMIT and
 * nothing is launched.  The first call on each device looks the array's address
 * up (the device on which the pointers live must be current, then and in every
 * later call) -- make that first call outside any stream capture and at
 * start-up: if nothing else of this library has run on the device yet, it is
 * also the moment the CUDA runtime loads the library's device code and reserves
 * the 8 MiB, which may synchronise the device and, on a GPU with no memory
 * left, fail.  Such a failure is returned as PSOPS_ECUDA (there is no context
 * to hold a message; cudaGetLastError has been cleared).  All calls on a device share the array and it is not cleared
 * between calls (every slot that is read has been written by the same call);
 * calls that overlap in time on one GPU overwrite each other's partial results,
 * so keep them on one stream or order them yourself.
 * Errors: EINVAL (also: a buffer that is host memory, or device memory of a GPU
 * other than the current one), EALIGN (a pointer not 4-byte aligned), ELIMIT,
 * ECUDA.
 */
#define PSOPS_STATIC_SCRATCH_DOUBLES (1 << 20)
int psops_quadratic_fitness_static(const float *d_x, int64_t ld, int32_t K, int64_t N,
                                   const float *d_dvec, const float *d_tvec,
                                   float *d_loss, void *cuda_stream);

/* Checkpoint / resume of the small state: the sync counter (kept on the
 * device, so both calls wait for the stream) and pBest_loss (host pointers, one
 * float per particle of the whole swarm).  x, v, pbest are the caller's own
 * tensors; with PSOPS_GBEST_HISTORY also move the remembered row and loss
 * (psops_get_history / psops_set_history).  Restoring these into a new context
 * on the same tensors continues the run bit for bit: the random stream is a
 * function of (seed, sync counter, particle, element) only. */
int psops_get_state(psops_ctx *ctx, uint32_t *sync_step, float *pbest_loss);
int psops_set_state(psops_ctx *ctx, uint32_t sync_step, const float *pbest_loss);

/* Inertia weight of Eq. 5 as psops_sync would compute it (host only). */
float psops_inertia(const psops_config *cfg, int64_t t_iter);

/* Number of kernel launches this context has enqueued so far. */
int64_t psops_launch_count(const psops_ctx *ctx);

/* Static description of an error code. */
const char *psops_strerror(int code);

/* Text of the last CUDA error seen by this context ("" if none). */
const char *psops_last_error(const psops_ctx *ctx);

/* Waits for the stream, then frees the context (not the caller's buffers). */
int psops_destroy(psops_ctx *ctx);

/*
 * ---------------------------------------------------------------------------
 * Operators of the training steps between two synchronisations
 *
 * A worker's local step needs the loss of its model (which at a sync point is
 * also the particle's fitness), the gradients, and an optimiser step.  The
 * operators below keep the conventions above: error codes, no device memory of
 * their own, a caller-owned 256-byte aligned workspace, work enqueued on the
 * context's stream, a context bound to the GPU current at creation and used by
 * one host thread at a time.  All of them are deterministic: the same inputs
 * give the same bits.  psops_*_set_stream moves a context to another stream of
 * its GPU: what it enqueues there comes after what it has enqueued so far (also
 * from one branch of a capture to another, but not into a capture or out of one,
 * where no such wait can be recorded: order the streams before the capture).  A
 * captured graph uses its context's workspace whenever it is replayed: order
 * replays and other calls of the context, and keep context and workspace for as
 * long as the graph.  Contexts are created outside captures (else ESTATE).
 * Arrays written on yet other streams are the caller's to order, as for any
 * kernel.  psops_*_destroy frees the context also where it returns an error.
 * ---------------------------------------------------------------------------
 */

/* element types */
#define PSOPS_NONE       0
#define PSOPS_F32        1
#define PSOPS_F16        2
#define PSOPS_BF16       3

/*
 * AdamW over many tensors in one launch.  Per element, with t the number of
 * the step (the first one after steps_done earlier steps is steps_done + 1):
 *   g  = grad * scale
 *   m' = m * beta1 + g * (1 - beta1)
 *   v' = v * beta2 + (g * g) * (1 - beta2)
 *   p' = p * (1 - lr * weight_decay)
 *        - (m' * (lr / (1 - beta1^t))) / (sqrt(v') * (1 / sqrt(1 - beta2^t)) + eps)
 * The factors in brackets are formed in double and rounded to fp32 once; every
 * operation on an element is fp32 round-to-nearest in the order written, each
 * product and sum rounded by itself (no fused multiply-add, correctly rounded
 * division and square root).
 *
 * state_bits 32: m and v are fp32.
 * state_bits 8: what is kept is m and the root r = sqrt(v) as 8-bit e4m3
 * numbers (no infinities, largest 448), with one fp32 scale for every 256
 * consecutive elements of a tensor (the last block of a tensor may be short):
 * value = number * scale, v = r * r.  The step itself uses the unrounded m'
 * and v'; then, per block with top = the largest magnitude,
 *   scale = top / 448,  number = round_to_nearest_even(value * (448 / top)),
 * a block with top < 2^-100 is kept as zeros with scale 0, and a root that is
 * not zero is never kept as zero (it becomes the smallest number), so that a
 * nonzero m never meets a vanished r.  Keeping the root halves the range that
 * 8 bits have to span.  A NaN or infinity in a gradient spoils its block.
 */
typedef struct {
    double   beta1, beta2;   /* in [0, 1)                                              */
    double   eps;            /* >= 0                                                   */
    int64_t  steps_done;     /* steps already taken (0 for a new run, t at resume)     */
    int32_t  state_bits;     /* 32 or 8                                                */
    int32_t  grad_type;      /* PSOPS_F32, PSOPS_F16, PSOPS_BF16                       */
    int32_t  copy_type;      /* PSOPS_NONE, PSOPS_F16, PSOPS_BF16: type of the copies  */
    int32_t  n_tensors;      /* >= 1                                                   */
} psops_adamw_config;

/* One parameter tensor: contiguous device arrays of n elements each. */
typedef struct {
    float   *p;              /* fp32 weights, e.g. a piece of a swarm's row            */
    const void *g;           /* gradient, grad_type                                    */
    void    *copy;           /* NULL, or n elements of copy_type that receive p'
                                (round to nearest): the weights a 16-bit model reads   */
    void    *m, *v;          /* fp32 m and v; or 8-bit m and r                         */
    float   *m_scale, *v_scale; /* 8 bits only: ceil(n / 256) fp32 scales each         */
    int64_t  n;              /* >= 0                                                   */
    double   weight_decay;
} psops_adamw_tensor;

typedef struct psops_adamw psops_adamw;  /* opaque */

/* Workspace for these tensors (only n is looked at); 0 if an argument is invalid. */
size_t psops_adamw_workspace_bytes(const psops_adamw_config *cfg, const psops_adamw_tensor *tensors);

/*
 * Adopts the caller's arrays (borrowed until psops_adamw_destroy; the list
 * itself is copied).  Tensors must not overlap.  Where all arrays of a tensor
 * lie alike within 8 elements (any view into flat buffers that are laid out the
 * same), whole groups of 8 elements move in one access; otherwise single
 * elements do, with the same results.
 * Errors: EINVAL, EALIGN (an array not aligned to its element), EWORKSPACE,
 * ENOMEM, ECUDA.  On error *out is NULL.
 */
int psops_adamw_create(psops_adamw **out, const psops_adamw_config *cfg, const psops_adamw_tensor *tensors,
                       void *d_workspace, size_t workspace_bytes, void *cuda_stream);

/* New gradient addresses, one per tensor (a framework that allocates gradients
 * anew for each step).  Enqueued on the stream: steps already enqueued keep the
 * old ones; the host waits for the table sent before, if that is still on its way.
 * EINVAL, EALIGN, ESTATE (inside a stream capture; nothing is changed), ECUDA. */
int psops_adamw_set_grads(psops_adamw *opt, const void *const *grads);

/*
 * One step.  d_scale: NULL (scale 1) or a device float that every gradient is
 * multiplied by (1 / loss scale, the clipping factor of psops_gradnorm, or
 * their product).  If *d_scale is not finite the step leaves everything as it
 * is and t does not advance.  t and the powers of beta live in device memory
 * and are advanced by the step itself, so a captured step can be replayed from
 * a CUDA graph (with the lr of the capture).
 * Errors: EINVAL (lr not finite), EALIGN, ECUDA.
 */
int psops_adamw_step(psops_adamw *opt, double lr, const float *d_scale);

/* t, read from the device (waits for the stream; ESTATE inside a stream capture). */
int psops_adamw_steps(psops_adamw *opt, int64_t *steps);

int psops_adamw_set_stream(psops_adamw *opt, void *cuda_stream);
int64_t psops_adamw_launch_count(const psops_adamw *opt);
const char *psops_adamw_last_error(const psops_adamw *opt);
int psops_adamw_destroy(psops_adamw *opt);   /* waits for the stream; frees nothing of the caller's */

/*
 * The 2-norm of many gradient tensors together and the factor that clips it:
 *   d_out[0] = norm = sqrt(sum of all squares)
 *   d_out[1] = min(1, max_norm / (norm + 1e-6)), or NaN if the norm is not
 *              finite (psops_adamw_step then skips the step)
 * Squares are fp32, eight of them (sixteen for 16-bit types) are added in fp32,
 * everything beyond in double, in a fixed order.  max_norm may be +inf (factor 1).
 * n[i] >= 0 elements at grads[i], contiguous.
 */
typedef struct psops_gradnorm psops_gradnorm;  /* opaque */
size_t psops_gradnorm_workspace_bytes(int32_t n_tensors, const int64_t *n);
int psops_gradnorm_create(psops_gradnorm **out, int32_t n_tensors, const void *const *grads, const int64_t *n,
                          int32_t grad_type, void *d_workspace, size_t workspace_bytes, void *cuda_stream);
int psops_gradnorm_set_grads(psops_gradnorm *gn, const void *const *grads);  /* as psops_adamw_set_grads */
int psops_gradnorm_run(psops_gradnorm *gn, float max_norm, float *d_out);
int psops_gradnorm_set_stream(psops_gradnorm *gn, void *cuda_stream);
int64_t psops_gradnorm_launch_count(const psops_gradnorm *gn);
const char *psops_gradnorm_last_error(const psops_gradnorm *gn);
int psops_gradnorm_destroy(psops_gradnorm *gn);

/*
 * Softmax cross entropy of a linear head over a large vocabulary, without
 * keeping the logits.  h: tokens x dim hidden states, w: vocab x dim weights
 * (both of one 16-bit type), targets: one label per token.
 *   logits[t, v] = sum_d h[t, d] w[v, d]
 *   lse[t]       = log sum_v exp(logits[t, v])
 *   rows[t]      = lse[t] - logits[t, targets[t]]
 *   loss         = sum_t rows[t] / n  (PSOPS_MEAN)  or  sum_t rows[t]  (PSOPS_SUM)
 * A token whose label lies outside [0, vocab) -- -100, say -- is left out: its
 * rows and lse are 0, it gets no gradient and gives none, whatever its hidden
 * state holds (NaN and infinities included); n counts the others.  With n = 0
 * the loss is 0.
 *   dlogits[t, v] = (exp(logits[t, v] - lse[t]) - [v == targets[t]]) * grad_t
 *   dh = dlogits w,  dw = dlogits^T h
 * with grad_t = *d_grad / n (PSOPS_MEAN), *d_grad (PSOPS_SUM) or d_grad[t]
 * (PSOPS_PER_TOKEN).  The gradient pass computes the logits once more, a piece
 * of the vocabulary at a time.  At a label the bracket is exp(-rows[t]) - 1; with
 * the rows of the forward pass at hand it keeps its digits where the token is
 * predicted with confidence, without them it is formed from the fp32 lse and
 * loses them as rows[t] goes below some 1e-3.
 *
 * Rounding: products are summed in fp32, softmax statistics are fp32, the loss
 * is summed in double.  The tensor cores cut sums off where fp32 would round to
 * nearest; they add up at most 768 terms of a logit and 8,192 of dh or dw in one
 * go, fp32 additions do the rest: 6e-5 of the largest partial sum at most in dh and
 * dw, however long the sum.  dlogits enters the two gradient products rounded to
 * the 16-bit type (that is what the tensor cores multiply), scaled by a power
 * of two that keeps small probabilities inside fp16's range; dh and dw are
 * rounded to the 16-bit type once, at the end.
 * Rows: row t of h, w, dh, dw starts at t * its stride (in elements, at least
 * dim).  dim a multiple of 8 with 16-byte aligned rows of w is read in place;
 * any other w, and any other dw, passes through the workspace
 * (PSOPS_XENT_STAGED), 512 MB of rows of each at a time.  dh and dw must not
 * overlap the inputs.
 * Should a product on the tensor cores ever wait in vain for its operands (four
 * seconds), the loss, the rows and lse of the tokens that count, dh and dw of
 * that call, and of every later call of the context that runs there, are NaN.
 */
#define PSOPS_MEAN       0
#define PSOPS_SUM        1
#define PSOPS_PER_TOKEN  2

#define PSOPS_XENT_GRADS   1u   /* reserve workspace for psops_xent_backward                    */
#define PSOPS_XENT_STAGED  2u   /* reserve workspace for rows of w / dw that are not 16-byte
                                   aligned although dim is a multiple of 8                      */

typedef struct {
    int64_t  max_tokens;     /* most tokens of a call, 1 .. 2^24                       */
    int64_t  dim;            /* 1 .. 2^20                                              */
    int64_t  vocab;          /* 1 .. 2^31 - 2^16                                       */
    int32_t  type;           /* PSOPS_F16 or PSOPS_BF16                                */
    uint32_t flags;
} psops_xent_config;

typedef struct psops_xent psops_xent;  /* opaque */

size_t psops_xent_workspace_bytes(const psops_xent_config *cfg);
int psops_xent_create(psops_xent **out, const psops_xent_config *cfg, void *d_workspace, size_t workspace_bytes,
                      void *cuda_stream);

/*
 * Loss only (the fitness of a worker's weights, or the first half of a training
 * step).  d_loss: one float (it can be the element of a device loss vector
 * given to psops_set_losses) or NULL; d_rows, d_lse: `tokens` floats each, or
 * NULL.  reduction: PSOPS_MEAN or PSOPS_SUM.  0 <= tokens <= max_tokens.
 * Errors: EINVAL, EALIGN (a pointer not aligned to its element; w not 16-byte
 * aligned without PSOPS_XENT_STAGED), ECUDA.
 */
int psops_xent_forward(psops_xent *x, const void *d_h, int64_t h_ld, const void *d_w, int64_t w_ld,
                       const int64_t *d_targets, int64_t tokens, int32_t reduction,
                       float *d_loss, float *d_rows, float *d_lse);

/*
 * Gradients, from the same h, w, targets and the lse of psops_xent_forward, and
 * its rows or NULL.
 * d_grad: the upstream gradient, see above.  d_dh or d_dw may be NULL (not
 * wanted).  Both are overwritten, not added to.  Errors: as forward, and ESTATE
 * without PSOPS_XENT_GRADS.
 */
int psops_xent_backward(psops_xent *x, const void *d_h, int64_t h_ld, const void *d_w, int64_t w_ld,
                        const int64_t *d_targets, int64_t tokens, const float *d_lse, const float *d_rows,
                        const float *d_grad, int32_t reduction,
                        void *d_dh, int64_t dh_ld, void *d_dw, int64_t dw_ld);

int psops_xent_set_stream(psops_xent *x, void *cuda_stream);
int64_t psops_xent_launch_count(const psops_xent *x);
const char *psops_xent_last_error(const psops_xent *x);
int psops_xent_destroy(psops_xent *x);

#ifdef __cplusplus
}
#endif
#endif /* PSOPS_H */
