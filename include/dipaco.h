/*
 * dipaco.h - C ABI of the module-wise outer synchronisation of DiPaCo on one CUDA device.
 *
 * The operation (DiPaCo, Algorithm 1, the outer-optimisation loop over levels and experts;
 * Sections 2.5-2.7).  A model is a grid of L levels with K_l modules per level (Section 2.2);
 * a path picks one module per level.  After the inner optimisation every path i holds its own
 * copy x_i of each module it passes through.  For every module (l,e):
 *
 *     Delta = sum_{i in R(l,e)} c_i * (theta - x_i)            outer gradient, Algorithm 1
 *     m'    = mu * m + Delta                                   Nesterov momentum (Section 2.5,
 *     theta'= theta - lr * (Delta + mu * m')                    lr/mu: supplementary details)
 *     x_i   = cast(theta')   for every path i through (l,e)    re-dispatch (Section 2.5)
 *
 * R(l,e) are the paths through (l,e) that reported this round (Section 2.6.2 trains subsets of
 * paths; Section 3.1 describes preempted workers); c_i = w_i / sum_{j in R} w_j with w the raw
 * per-path weights (shard sizes, Section 2.7 "Loss reweighing"; uniform when absent).  A module
 * with no reporting path, or zero total weight, keeps theta and m bit for bit; its copies are
 * still overwritten with cast(theta).  The reduction runs in ascending path id in fp32 with
 * fused multiply-adds, so results are bitwise reproducible and identical between the resident
 * and the chunked mode.
 *
 * Layouts.  theta and momentum: fp32, sum_l K_l*N_l elements ordered [level][module][element]
 * (N_l = |B_l|, the size of every module of level l).  A path copy: sum_l N_l elements, the
 * path's L modules concatenated in level order, fp32 or bf16 (round-to-nearest-even on write).
 *
 * Ownership.  The caller owns theta, momentum and all path buffers; they are updated in place.
 * A context owns small device tables and, in chunked mode, an fp32 partial-sum scratch.
 *
 * Errors.  Every function returns a status (0 = ok, negative = error) and never throws, aborts
 * or prints.  Arguments are validated before anything is launched: on a validation error the
 * caller's buffers are untouched.  Calls are asynchronous on the given stream unless noted; all
 * calls on one context must be ordered on one stream (or externally synchronised).
 */
#ifndef DIPACO_H
#define DIPACO_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct dipaco_ctx dipaco_ctx;

enum { DIPACO_F32 = 0, DIPACO_BF16 = 1 };

enum {
    DIPACO_OK = 0,
    DIPACO_EINVAL = -1,   /* bad argument (null, out of range, non-finite, wrong state value)   */
    DIPACO_ECUDA = -2,    /* a CUDA runtime call failed                                         */
    DIPACO_ENOMEM = -3,   /* host or device allocation failed                                   */
    DIPACO_ESTATE = -4,   /* call not allowed in the context's current state                    */
    DIPACO_ETIMEOUT = -5, /* a bounded wait inside a kernel ran out (reported by device_status) */
    DIPACO_ENODEV = -6,   /* the context was created without a device (plan only)               */
    DIPACO_ELIMIT = -7    /* a size exceeds a fixed limit of the entry point (static scratch)   */
};

/* outer optimisers for dipaco_set_optimizer */
enum {
    DIPACO_OPT_NESTEROV = 0, /* m' = mu*m + Delta; theta' = theta - lr*(Delta + mu*m')   (the paper's) */
    DIPACO_OPT_MOMENTUM = 1, /* m' = mu*m + Delta; theta' = theta - lr*m'                (heavy ball)  */
    DIPACO_OPT_SGD = 2,      /* theta' = theta - lr*Delta; momentum left as it is (lr = 1: averaging)   */
    DIPACO_OPT_ADAM = 3      /* Adam family, configured by dipaco_set_adam                              */
};

/* what the path buffers hold on entry, for dipaco_set_input_kind */
enum {
    DIPACO_INPUT_COPIES = 0,   /* each path's copy x_i of its modules: Delta = sum c_i (theta - x_i)  */
    DIPACO_INPUT_GRADIENTS = 1 /* each path's gradient g_i of its modules: Delta = sum c_i g_i         */
};

/* kernel selection for dipaco_set_kernel */
enum {
    DIPACO_KERNEL_AUTO = 0,   /* bulk-copy (TMA) pipeline, one element per thread for the few elements
                                 before and after its range                                            */
    DIPACO_KERNEL_VECTOR = 1, /* 128-bit register loads/stores on whole steps, one element per thread
                                 for the rest                                                         */
    DIPACO_KERNEL_SCALAR = 2  /* one element per thread everywhere                                    */
};
/*
 * Alignment.  Nothing has to be aligned beyond its element size.  Path copies may start at any
 * element boundary, each at its own, and level sizes may be odd (modules and slots then start
 * inside 16-byte units): the bulk-copy and the vector kernel each have a variant that loads the
 * aligned 16-byte units around the data and writes realigned units, at 0.91-0.95 of the speed of
 * fully aligned buffers (bulk-copy kernel).  They need theta, momentum (and the second moment) to
 * sit at the same place within a 16-byte unit, which holds whenever these arrays are allocated the
 * same way; otherwise the module falls back to one element per thread.
 */

/*
 * Build a context for one module grid (Algorithm 1, "Require" lines; Section 2.2 notation).
 *   num_levels         L >= 1
 *   modules_per_level  host [L], K_l >= 1
 *   level_numel        host [L], N_l >= 0
 *   num_paths          P >= 1; any set of paths, not only the full product (Section 2.6.2)
 *   path_to_module     host [P*L] row-major, entry (i,l) in [0,K_l); a module no path uses is
 *                      allowed and never touched (Section 2.6.1: any sharing pattern)
 *   path_weights       host [P] raw weights >= 0, finite (Section 2.7), or NULL = uniform
 *   outer_lr, outer_momentum   finite; the paper uses 0.7 and 0.9
 *   path_dtype         DIPACO_F32 or DIPACO_BF16
 *   chunk_paths        0 = all path copies are resident at once; c > 0 = copies are presented
 *                      in chunks of c consecutive path ids (Section 3.3, online averaging)
 *   device             CUDA device ordinal, or -1 for a plan-only context (no CUDA call is made;
 *                      only the dipaco_plan_* queries work, everything else returns ENODEV)
 * All host arrays are copied.  Synchronous.
 */
int dipaco_create(dipaco_ctx **out, int32_t num_levels, const int32_t *modules_per_level,
                  const int64_t *level_numel, int32_t num_paths, const int32_t *path_to_module,
                  const float *path_weights, float outer_lr, float outer_momentum,
                  int32_t path_dtype, int32_t chunk_paths, int32_t device);

/*
 * One outer synchronisation of every module, in place (Algorithm 1, outer loop, plus re-dispatch).
 *   theta, momentum  device, fp32, layout above; in/out
 *   path_ptrs        HOST array [P] of DEVICE pointers, one per path copy; in/out
 *   reported         HOST [P], nonzero = path i reported; NULL = all reported
 *   cuda_stream      a cudaStream_t (0 = default stream)
 * With chunk_paths = 0 this is one fused pass; otherwise the library walks the chunks in
 * ascending order over the same device pointers, one launch per chunk, carrying fp32 partial
 * sums; the launch that sees a module's last reporting path finishes the module and writes
 * cast(theta') into all of its paths.  A call with the same settings, buffers and mask as the
 * previous one on this context reuses that call's plan and device tables: it only launches
 * kernels (no upload, no allocation, no synchronisation), so it may be recorded in a CUDA graph
 * by stream capture once one ordinary call has planned it.  Replaying the graph is then the
 * cheapest way to repeat a small synchronisation (2x2 grid: 5.5 us per replayed call against
 * 8.2 us per launched call).  Any dipaco_set_* call, another mask or other buffers make the next
 * call plan and upload again, which must not happen during capture.
 */
int dipaco_outer_sync(dipaco_ctx *ctx, float *theta, float *momentum, void *const *path_ptrs,
                      const uint8_t *reported, void *cuda_stream);

/*
 * Incremental form of the same operation for callers that hold only one chunk of path copies
 * on the device at a time (Section 3.3, "Online Parameter Gradient Averaging": each checkpoint
 * is added to a partial sum as it arrives).  Requires chunk_paths > 0.  Chunk c covers path ids
 * [c*chunk_paths, min(P, (c+1)*chunk_paths)).
 *   begin      fixes theta, momentum, the mask and the stream for this round.
 *   accumulate chunk_index must be 0,1,2,... in order; chunk_ptrs is a HOST array of the
 *              chunk's DEVICE pointers.  Adds the chunk's reporting copies to the partial sums;
 *              a module whose last reporting path lies in this chunk is updated right away and
 *              written into this chunk's copies.
 *   writeback  after every chunk has been accumulated, any order: fills every slot of the
 *              chunk's copies with cast(theta') (the contents of chunk_ptrs are not read, so the
 *              buffers may be fresh).
 *   end        checks that every chunk was accumulated and returns the context to idle.
 * With bf16 copies the first begin on a context allocates a scratch of 2 bytes per module
 * parameter: the finishing passes store cast(theta') there and the write-back launches read it
 * instead of fp32 theta'.  If that allocation fails the write-back reads theta' (same results).
 */
int dipaco_sync_begin(dipaco_ctx *ctx, float *theta, float *momentum, const uint8_t *reported,
                      void *cuda_stream);
int dipaco_sync_accumulate(dipaco_ctx *ctx, int32_t chunk_index, void *const *chunk_ptrs);
int dipaco_sync_writeback(dipaco_ctx *ctx, int32_t chunk_index, void *const *chunk_ptrs);
int dipaco_sync_end(dipaco_ctx *ctx);

/*
 * The same synchronisation for state that lives in HOST memory (checkpoints that do not fit
 * on the device; Section 3.3: the executor loads checkpoints and averages them as they come):
 * theta, momentum [module params] and the P path copies are host buffers (pinned memory gives
 * full copy speed).  The work is streamed through the device slab by slab: an element range of
 * one module together with that range of every reporting copy is uploaded, reduced, updated and
 * cast in one fused pass, and the result is copied back into theta, momentum and the slot of
 * every path of the module while the next slab is already being uploaded.  Device staging is
 * bounded by the size of chunk_paths path copies (> 0 required) plus theta and momentum.  Paths
 * that did not report are not uploaded.  Path copies that lie equally spaced in host memory
 * (rows of one allocation) are moved with one strided copy per slab instead of one per path.
 * By default a pool of host threads fans each module's result out to its paths
 * (dipaco_set_host_threads).  Results are bitwise those of dipaco_outer_sync.  Synchronous: returns when all host buffers
 * hold the result, and on an error only after every copy it started has finished.
 */
int dipaco_outer_sync_host(dipaco_ctx *ctx, float *theta_host, float *momentum_host,
                           void *const *path_ptrs_host, const uint8_t *reported,
                           void *cuda_stream);

/* Replace the raw per-path weights (host [P], or NULL = uniform).  Section 2.7. */
int dipaco_set_weights(dipaco_ctx *ctx, const float *path_weights);

/*
 * Outer gradient norm rescaling (Section 2.7): the finished outer gradient of module (l,e) is
 * multiplied by module_scale[(l,e)] before the optimiser step, Delta <- s * Delta.  host
 * [sum_l K_l], level-major, finite; NULL = no rescaling.  The paper rescales by the square root
 * of the number of paths through the module; the factor itself (sqrt(P) or its inverse) is the
 * caller's to supply.  A factor of exactly 1 leaves the result bit-identical.
 */
int dipaco_set_module_scale(dipaco_ctx *ctx, const float *module_scale);

/*
 * Levels that take no part in the exchange (Section 4.2: in the models with path-specific
 * modules some blocks stay local to their path): host [L], 0 = theta, momentum and every copy
 * of the level's modules are left untouched; NULL = every level is synchronised.
 */
int dipaco_set_level_sync(dipaco_ctx *ctx, const uint8_t *level_sync);

/*
 * Outer optimiser (Section 2.5: Nesterov momentum is the paper's choice; other optimisers of the
 * federated family fit the same scheme).  DIPACO_OPT_*; the default is Nesterov.
 */
int dipaco_set_optimizer(dipaco_ctx *ctx, int32_t optimizer);

/*
 * Adam-family optimiser.  It covers the adaptive federated optimisers that Section 2.5 names as
 * alternatives (step = 0: no bias correction, eps plays the role of their adaptivity constant)
 * and the AdamW of the fully synchronous ablation of Section 4.5 (step = t >= 1: bias-corrected,
 * decoupled weight decay).  With Delta the module's outer gradient, the `momentum` argument of
 * the sync calls as first moment m and second_moment as v:
 *     m' = b1*m + (1-b1)*Delta        v' = b2*v + (1-b2)*Delta^2
 *     theta' = theta*(1 - lr*weight_decay) - lr * (m'/c1) / (sqrt(v'/c2) + eps)
 *     c1 = 1 - b1^step, c2 = 1 - b2^step   (both 1 when step = 0)
 * second_moment: device, fp32, same layout as theta, caller-owned, in/out.  0 <= b1, b2 < 1,
 * eps >= 0.  Selects DIPACO_OPT_ADAM; call again to advance `step`.  The outer_momentum given at
 * create is not used.  second_moment lives where theta lives: a device array for
 * dipaco_outer_sync and the chunk API, a host array for dipaco_outer_sync_host.
 */
int dipaco_set_adam(dipaco_ctx *ctx, float *second_moment, float beta1, float beta2, float eps,
                    float weight_decay, int32_t step);

/*
 * What the path buffers hold on entry (DIPACO_INPUT_*).  With gradients the reduction is the
 * module-by-module gradient aggregation of Section 4.5; the buffers are still overwritten with
 * cast(theta') on exit, so after the call every path holds the new parameters of its modules.
 */
int dipaco_set_input_kind(dipaco_ctx *ctx, int32_t input_kind);

/*
 * Sharded executor (Section 3.3, "Sharded Outer Optimization Executor": modules, and the
 * parameters inside a module, are independent, so the update can be split over executors with no
 * exchange between them).  This context then owns slab shard_index of shard_count of EVERY
 * module (equal element ranges cut at multiples of 8192 elements; the last shard takes the
 * remainder) and touches nothing else: theta, momentum and the path copies outside its slabs are
 * neither read nor written.  Pointers and layouts stay those of the whole problem, so S contexts
 * (one per GPU, each holding at least its slabs at the usual offsets) together perform exactly
 * the unsharded update, bit for bit.  Default: shard 0 of 1.
 */
int dipaco_set_shard(dipaco_ctx *ctx, int32_t shard_index, int32_t shard_count);

/*
 * The same partition for executors that hold ONLY their slab (Section 3.3: each executor of the
 * sharded outer optimiser owns a part of the parameters and the matching part of every
 * checkpoint).  Every module of level l has N_l elements, so shard s of S owns the same element
 * range [begin_l, end_l) of every module of that level; dipaco_plan_shard returns it (host only,
 * works on plan-only contexts).  Ranges are cut at multiples of 8192 elements, the last shard
 * takes the remainder; over s = 0..S-1 they tile [0, N_l) exactly once.
 */
int dipaco_plan_shard(const dipaco_ctx *ctx, int32_t shard_index, int32_t shard_count, int32_t level,
                      int64_t *begin, int64_t *end);

/*
 * A context for shard shard_index of shard_count of the problem that `whole` describes, in the
 * compact layout: the shard is itself a module grid with the same levels, modules, paths and
 * weights and with N_l replaced by end_l - begin_l.  Its theta, momentum (and second moment)
 * hold, module after module, elements [begin_l, end_l) of each module; its path copies hold,
 * level after level, elements [begin_l, end_l) of the path's slot: each executor allocates 1/S
 * of everything and no pointer to the rest is ever needed.  Every entry point works on it as on
 * any context, and the S results, put back side by side, are bit for bit the unsharded update:
 * no exchange between executors (elements are independent).  The new context copies the
 * weights, module scales, level flags, learning rate, momentum, optimiser, input kind, chunk
 * size, kernel choice and tuning of `whole` as they are at the time of the call (`whole` may be
 * plan-only and may be destroyed afterwards); the Adam family must be selected on the shard
 * itself with dipaco_set_adam, because it needs the shard's own second-moment array.
 * device: CUDA device of this executor, or -1 for plan only.
 */
int dipaco_create_shard(dipaco_ctx **out, const dipaco_ctx *whole, int32_t shard_index,
                        int32_t shard_count, int32_t device);

/* Choose the kernel family (DIPACO_KERNEL_*); all families give bitwise identical results. */
int dipaco_set_kernel(dipaco_ctx *ctx, int32_t kernel);

/*
 * Tuning of the bulk-copy kernel: persistent CTAs per SM (1..8), pipeline depth in tiles (2..32),
 * 16-byte units of path data per compute thread and tile (1, 2 or 4; the tile is
 * 256 threads * units * 16 bytes) and the number of theta/momentum/result tile buffers (2..4;
 * more of them help modules with few contributors).  0 keeps a value.  A depth that does not fit
 * the shared memory of the chosen layout is rejected with DIPACO_EINVAL and nothing changes;
 * result buffers beyond two are dropped at launch while they would leave the ring shallower than a
 * launch of that mix of modules needs (10 stages when most elements have 8 or more contributors,
 * 6 otherwise).  A launch that stages more fp32 tiles per buffer than the layout was accepted
 * for (the second moment of an Adam-family optimiser selected later) falls back to the next
 * smaller tile that fits; results do not depend on any of this.
 */
int dipaco_set_tuning(dipaco_ctx *ctx, int32_t ctas_per_sm, int32_t stages,
                      int32_t units_per_thread, int32_t io_slots);

/*
 * Tuning of the bulk-copy kernel's dynamic scheduling: a launch is cut into work items (runs of
 * tiles of one module) that the persistent CTAs draw from a counter.  An item moves at most
 * max_item_bytes of traffic (default 2 MiB) and a launch is cut into at least items_per_cta
 * items per CTA (default 64) so that the CTAs finish together.  0 keeps a value.  Results do not
 * depend on the cut.
 */
int dipaco_set_work_items(dipaco_ctx *ctx, int64_t max_item_bytes, int32_t items_per_cta);

/*
 * Tuning of dipaco_outer_sync_host: the most bytes of path data that one streamed unit stages
 * on the device in each direction (0 = the default, 512 MiB; always at least one tile of every
 * copy of the module, at most 1/6 of chunk_paths path copies).  The download of a unit cannot
 * start before the unit is uploaded and reduced, so a call takes about one unit's transfer time
 * longer than the PCIe transfer itself: smaller units shorten that, larger ones mean fewer and
 * larger copies.
 */
int dipaco_set_host_unit_bytes(dipaco_ctx *ctx, int64_t bytes);

/*
 * Host threads of dipaco_outer_sync_host.  Every path of a module receives the same
 * cast(theta'), so with threads > 0 each streamed piece of it is downloaded once, into a pinned
 * buffer of the library, and `threads` host threads copy it into the slot of every path while
 * later pieces are still being uploaded: PCIe carries one copy per module instead of one per
 * path.  The threads belong to the context (created by the first call that needs them, joined
 * by dipaco_destroy) and sleep between calls.  0 = no host threads: the device writes one copy
 * per path and all of them are downloaded.  -1 = the default (half the hardware threads, at
 * most 4: more of them compete with the uploads for host memory bandwidth).  Results are
 * identical either way.
 */
int dipaco_set_host_threads(dipaco_ctx *ctx, int32_t threads);

/*
 * Synchronise the context's last stream and report what the kernels recorded: DIPACO_OK, or
 * DIPACO_ETIMEOUT if a bounded wait gave up, or DIPACO_ECUDA.  Clears the recorded status.
 *
 * Every wait inside the kernels is bounded (4 s).  A kernel whose wait runs out records a code
 * in the context's error word and ends in an orderly way (copies in flight are waited for); the
 * results of that call are undefined.  The error is sticky on the device: every later launch on
 * the context sees the error word set and does nothing at all (buffers untouched, status of the
 * entry point still DIPACO_OK since launches are asynchronous) until this function has been
 * called; it returns DIPACO_ETIMEOUT once, re-arms the context (error word and work counters
 * back to zero) and from then on calls work again.
 */
int dipaco_device_status(dipaco_ctx *ctx);

/*
 * Diagnostic: make a bounded wait run out on purpose, harmlessly.  Launches one warp on the
 * given stream whose first thread waits at most limit_ns (1 .. 1e9) on a barrier that nothing
 * will complete; no copy is in flight and no buffer of the caller is involved.  When the wait
 * gives up the kernel leaves what a pipeline kernel that gave up leaves: a code in the error
 * word and a work counter that is not back at zero.  Afterwards the context behaves as after a
 * real time-out (see dipaco_device_status).  Lets an application or a test check its handling of
 * DIPACO_ETIMEOUT.  The paper has no counterpart.
 */
int dipaco_selftest_wait_expiry(dipaco_ctx *ctx, int64_t limit_ns, void *cuda_stream);

/* Number of kernels this context has launched so far. */
int64_t dipaco_launch_count(const dipaco_ctx *ctx);

/*
 * Plan queries (host only; work on plan-only contexts too).  They expose the host-side
 * decisions: the contributor set of a module under a mask and the normalised coefficients.
 *   members / contributors  out, capacity num_paths each; ascending path ids
 *   coeff                   out, capacity num_paths; c_i as the kernels use them (fp32)
 *   will_update             out; 0 when no path reports or the total weight is zero
 * Any out pointer may be NULL.
 */
int dipaco_plan_module(const dipaco_ctx *ctx, int32_t level, int32_t module,
                       const uint8_t *reported, int32_t *num_members, int32_t *members,
                       int32_t *num_contributors, int32_t *contributors, float *coeff,
                       int32_t *will_update);
/* Offsets (in elements) of module (level, module) in theta and of the level in a path copy. */
int dipaco_plan_offsets(const dipaco_ctx *ctx, int32_t level, int32_t module,
                        int64_t *theta_offset, int64_t *path_offset, int64_t *numel);
/* Number of chunks (1 when chunk_paths = 0) and fp32 elements of partial-sum scratch. */
int dipaco_plan_chunks(const dipaco_ctx *ctx, int32_t *num_chunks, int64_t *scratch_elems);

/*
 * Bytes that one dipaco_outer_sync on this context moves through device memory by
 * construction (every read and write of theta, momentum, partial sums and path copies, summed
 * over its launches), and the number of launches (tail launches not counted).  For a resident
 * context this is the algorithmic minimum; for a chunked one it includes the partial-sum traffic.
 */
int dipaco_plan_traffic(const dipaco_ctx *ctx, const uint8_t *reported, int64_t *bytes,
                        int32_t *launches);

/*
 * The split of the resident-mode launch over num_ctas persistent CTAs in tiles of `tile`
 * elements (all pointers assumed aligned): CTA b processes segments
 * [cta_first[b], cta_first[b+1]); segment s covers elements [seg_begin[s], seg_end[s]) of
 * module (seg_level[s], seg_module[s]).  Arrays have `capacity` entries (cta_first: num_ctas+1).
 * Returns the number of segments (>= 0), or a negative status (EINVAL also when capacity is
 * too small).
 */
int dipaco_plan_split(const dipaco_ctx *ctx, const uint8_t *reported, int32_t num_ctas, int64_t tile,
                      int32_t capacity, int32_t *seg_level, int32_t *seg_module, int64_t *seg_begin,
                      int64_t *seg_end, int32_t *cta_first);

int dipaco_destroy(dipaco_ctx *ctx);

/*
 * Synchronise ONE module without allocating anything.  (The paper has no counterpart for this
 * entry point; it exists for the sake of its callers.)
 *
 * Who needs it: code that is not allowed to touch the device allocator.  Examples are a process
 * that has handed all device memory to a pool of its own at start-up, so that a later cudaMalloc
 * simply fails, and a latency-critical loop that cannot accept the device-wide synchronisation
 * that cudaMalloc and cudaFree imply.  Such callers cannot use dipaco_create (it allocates
 * tables, and in chunked mode the partial-sum scratch).  This function takes everything as
 * arguments, passes the per-chunk tables inside the kernel arguments and keeps the partial sums
 * in a static device array that is part of the library image.  It calls no cudaMalloc, cudaFree,
 * cudaMallocHost or any other allocating routine, on the device or on the host heap.
 *
 * What it computes: the same result, bit for bit, as dipaco_outer_sync on a grid with a single
 * level and a single module shared by num_paths paths, walked in chunks of chunk_paths.
 *   theta, momentum   device, fp32 [numel]; in/out
 *   numel             0 <= numel <= DIPACO_STATIC_MAX_NUMEL (4 Mi parameters = 16 MiB of partial
 *                     sums); larger sizes are refused with DIPACO_ELIMIT and nothing is launched
 *   num_paths         >= 1
 *   copy_ptrs         HOST array [num_paths] of DEVICE pointers, each a copy of the module
 *                     ([numel] of path_dtype); in/out, every copy is overwritten with cast(theta')
 *   path_weights      HOST [num_paths] raw weights >= 0 or NULL = uniform
 *   reported          HOST [num_paths], nonzero = reported, or NULL = all
 *   chunk_paths       1..32 copies per chunk
 *   device            CUDA device that owns all the buffers; made current during the call
 *   cuda_stream       stream the kernels are launched on (asynchronous)
 *
 * The static array: 16 MiB per GPU.  It is part of the library's CUDA module, so the CUDA runtime
 * reserves it when it loads that module on a GPU: with lazy module loading (the default) that is
 * the first call of this function on the device, with eager loading the creation of the context.
 * From then on the GPU holds the 16 MiB until the process exits, whether or not this function is
 * called again.  The first call on a device (any numel >= 1) is therefore the set-up call: make
 * it while the device still has room for the module (a caller that gives all device memory to
 * its own pool makes it before that), and before any stream capture begins; if the module cannot
 * be loaded it returns DIPACO_ENOMEM (or DIPACO_ECUDA), launches nothing and leaves no CUDA error
 * pending.  Every call looks the array's device address up again (cudaGetSymbolAddress: no
 * allocation once the module is loaded).  All calls on one device share the array and it keeps
 * whatever the last call left in it: each call starts its sums from zero in the kernel, so stale
 * contents are never read, but two calls that overlap on the GPU (different streams, or
 * different host threads) race on it and must be serialised by the caller.
 */
#define DIPACO_STATIC_MAX_NUMEL (4 * 1024 * 1024)
int dipaco_module_sync_static(float *theta, float *momentum, int64_t numel, int32_t num_paths,
                              void *const *copy_ptrs, const float *path_weights,
                              const uint8_t *reported, float outer_lr, float outer_momentum,
                              int32_t path_dtype, int32_t chunk_paths, int32_t device,
                              void *cuda_stream);

/*
 * Operators of the inner phase.  Between two synchronisations every path is trained on its own shard
 * (Algorithm 1, the inner-optimisation loop).  With the copies of hundreds of paths resident little
 * device memory is left for activations, so the operators below keep activations in 8 bits: a block
 * of a path runs its norm, its products and its activation on them, forward and backward, and hands
 * gradients to an inner optimiser.  They need no context: every buffer is an argument.
 *
 * Conventions.  All pointers are device pointers; the calls are asynchronous on cuda_stream, allocate
 * nothing and can be captured in a CUDA graph.  Arguments are checked before anything is launched
 * (DIPACO_EINVAL, or DIPACO_ELIMIT for extents of about 2^31 and more).  A dense matrix is row-major
 * with a row stride in elements, at any element alignment; 16-byte aligned rows are fastest.  Rows at
 * other alignments are read in the aligned 16-byte units that hold their values, except by the forward
 * norm, which reads and writes them value by value unless both x and y are aligned.  dtype and
 * param_dtype are DIPACO_F32 or DIPACO_BF16.  Outputs must not overlap inputs.  Extents of zero are
 * allowed.  Every sum is fp32 and taken in an order that depends on shapes, types and alignment alone:
 * results are bitwise reproducible.
 *
 * Packed matrices.  8-bit codes (e4m3: 4 exponent and 3 mantissa bits, largest value 448, no infinity)
 * with one scale for each block of 128 x 128 values, itself an 8-bit power of two (e8m0: byte b is
 * 2^(b-127), 255 is NaN): value = code * scale.  Packing takes the least scale that brings the largest
 * finite magnitude of the block to at most 448 (at least 2^-126; a block of zeros has scale 1) and
 * rounds to the nearest code, ties to even; an infinity or NaN becomes a NaN code and does not
 * influence the scale.  Blocks are square so that the scale is constant over 128 contracted values
 * along either side: the same bytes serve a product, its input gradient and its weight gradient.
 *   codes   rows x cols bytes, row stride `stride` bytes; 16-byte aligned, stride a multiple of 16
 *   scales  [ceil(rows/128)][ceil(cols/128)] bytes, row-major
 */
typedef struct dipaco_packed {
    void *codes;
    void *scales;
    int64_t rows, cols, stride;
} dipaco_packed;

/* Dense to packed, and back (a code times its scale, rounded once to dtype: an infinity for 2^128, to which
 * magnitudes near the largest fp32 value round). */
int dipaco_pack(const void *x, int64_t x_stride, int32_t dtype, const dipaco_packed *out, int32_t device,
                void *cuda_stream);
int dipaco_unpack(const dipaco_packed *x, void *y, int64_t y_stride, int32_t dtype, int32_t device,
                  void *cuda_stream);

/*
 * Layer norm of every row:  mean = sum x / C,  var = sum (x - mean)^2 / C,
 * rstd = 1 / sqrt(var + eps),  y = (x - mean) * rstd * gamma + beta.
 *   gamma, beta  [cols] of param_dtype; NULL = ones, zeros
 *   y            NULL = statistics only
 *   mean, rstd   [rows] fp32, kept for the backward pass; NULL where not wanted; NaN for rows of no values
 */
int dipaco_layer_norm(const void *x, int64_t x_stride, const void *gamma, const void *beta, void *y,
                      int64_t y_stride, float *mean, float *rstd, int64_t rows, int64_t cols, float eps,
                      int32_t dtype, int32_t param_dtype, int32_t device, void *cuda_stream);

/*
 * The same with the result packed straight from its fp32 value (it feeds a product) and, unless
 * x_packed is NULL, the input packed as the checkpoint that dipaco_layer_norm_backward reads.  The
 * extents are those of y; mean and rstd are required and come from the exact input.
 */
int dipaco_layer_norm_pack(const void *x, int64_t x_stride, const void *gamma, const void *beta,
                           const dipaco_packed *y, const dipaco_packed *x_packed, float *mean, float *rstd,
                           float eps, int32_t dtype, int32_t param_dtype, int32_t device, void *cuda_stream);

/*
 * Gradient of the layer norm.  With h = (x - mean) * rstd and g = dy * gamma:
 *   dx = rstd * (g - mean(g) - h * mean(g h)),  dgamma = sum over rows of dy h,  dbeta = sum of dy.
 *   x, x_packed    exactly one of them: the input, or its 8-bit checkpoint
 *   gamma          NULL = ones
 *   dx             of dtype (that of dy and of a dense x); dgamma, dbeta [cols] fp32, overwritten
 *                  (zero for no rows); each may be NULL, not all three
 *   workspace      16-byte aligned, at least the bytes that dipaco_layer_norm_workspace reports (a
 *                  host-only query; may be zero); not needed without dgamma and dbeta
 */
int dipaco_layer_norm_workspace(int64_t rows, int64_t cols, int64_t *bytes);
int dipaco_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                               const dipaco_packed *x_packed, const float *mean, const float *rstd,
                               const void *gamma, void *dx, int64_t dx_stride, float *dgamma, float *dbeta,
                               int64_t rows, int64_t cols, int32_t dtype, int32_t param_dtype, void *workspace,
                               int64_t workspace_bytes, int32_t device, void *cuda_stream);

/*
 * The norms after and before a block with its gate and its scaled residual, for a block's result f and the
 * residual stream x, LN being the norm above without parameters:
 *   p = LN(f) post_gamma + post_beta   (p = f without post_norm)
 *   z = residual_scale x + gate p      (rounded to dtype: what the stream holds)
 *   n = LN(z) gamma + beta             (of the z that the stream holds; not computed without norm)
 *   gate           DIPACO_GATE_NONE (1), or one gate for a column ([cols]), a row ([rows]) or a value ([rows,
 *                  cols] with row stride gate_stride, of dtype); [cols] and [rows] of gate_dtype
 *   gamma, beta, post_gamma, post_beta   [cols] of param_dtype; NULL = ones, zeros; none without their norm
 *   stats          [4][rows] fp32, kept for the backward pass: mean and rstd of f, mean and rstd of z; 0 and 1
 *                  for a norm that is left out, NaN for rows of no values
 */
enum { DIPACO_GATE_NONE = 0, DIPACO_GATE_COLS = 1, DIPACO_GATE_ROWS = 2, DIPACO_GATE_FULL = 3 };
typedef struct dipaco_residual_norm_args {
    int64_t rows, cols;
    const void *gamma, *beta, *post_gamma, *post_beta, *gate;
    int64_t gate_stride;
    int32_t gate_kind, gate_dtype, dtype, param_dtype;
    int32_t post_norm, norm;  /* nonzero: with that norm */
    float residual_scale, eps;
} dipaco_residual_norm_args;

/* n is dense (n; NULL = statistics only) or packed (n_packed), with z packed as a checkpoint beside it unless z_packed is
 * NULL; z itself is always written. */
int dipaco_residual_norm(const dipaco_residual_norm_args *args, const void *x, int64_t x_stride, const void *f,
                         int64_t f_stride, void *z, int64_t z_stride, void *n, int64_t n_stride,
                         const dipaco_packed *n_packed, const dipaco_packed *z_packed, float *stats, int32_t device,
                         void *cuda_stream);

/*
 * Gradients from those of n (dn; with norm only) and z (dz; NULL = none).  With h = (v - mean) rstd of z or f:
 *   d = dz + rstd_z (u - mean(u) - h_z mean(u h_z)),  u = dn gamma;   dx = residual_scale d
 *   df = rstd_f (q - mean(q) - h_f mean(q h_f)),  q = d gate post_gamma   (q itself without post_norm)
 *   dgate = d p, summed over what shares a gate;  dpost_gamma = sum d gate h_f,  dpost_beta = sum d gate,
 *   dgamma = sum dn h_z,  dbeta = sum dn, over rows (a gate of columns is multiplied with post_gamma, and with the
 *   sums, so that q and the sums overflow where those products do)
 *   f or f_packed, z or z_packed   exactly one of each: the forward call's, or 8-bit checkpoints of them (z with norm
 *                  only)
 *   dx, df         of dtype; NULL where not wanted, as the following
 *   dgate          [cols] or [rows] fp32, or [rows, cols] of dtype with row stride dgate_stride
 *   dgamma ...     [cols] fp32; overwritten, zero for no rows
 *   workspace      16-byte aligned, at least the bytes that dipaco_residual_norm_workspace reports (host only)
 */
int dipaco_residual_norm_workspace(int64_t rows, int64_t cols, int64_t *bytes);
int dipaco_residual_norm_backward(const dipaco_residual_norm_args *args, const void *dn, int64_t dn_stride, const void *dz,
                                  int64_t dz_stride, const void *f, int64_t f_stride, const dipaco_packed *f_packed,
                                  const void *z, int64_t z_stride, const dipaco_packed *z_packed, const float *stats,
                                  void *dx, int64_t dx_stride, void *df, int64_t df_stride, void *dgate,
                                  int64_t dgate_stride, float *dgamma, float *dbeta, float *dpost_gamma,
                                  float *dpost_beta, void *workspace, int64_t workspace_bytes, int32_t device,
                                  void *cuda_stream);

/*
 * GELU in its tanh form, gelu(x) = x * s with s = 1 / (1 + exp(-2u)), u = sqrt(2/pi) (x + 0.044715 x^3),
 * packed from its fp32 value, and, unless x_packed is NULL, its input packed as a checkpoint.
 * The backward call reads that checkpoint and packs dy * gelu'(x) for the two products that follow,
 * gelu'(x) = s + x s (1 - s) 2u'.  An infinite input gives NaN, like its product 0 * infinity.
 */
int dipaco_gelu_pack(const void *x, int64_t x_stride, int32_t dtype, const dipaco_packed *y,
                     const dipaco_packed *x_packed, int32_t device, void *cuda_stream);
int dipaco_gelu_pack_backward(const void *dy, int64_t dy_stride, int32_t dtype, const dipaco_packed *x_packed,
                              const dipaco_packed *dx, int32_t device, void *cuda_stream);

/*
 * Product of two packed matrices on the tensor cores, C = op(A) op(B) with fp32 sums, rounded once to
 * dtype.  The tensor cores truncate when they add, 32 products at a time: each product to 2^-25 of the sum
 * so far, and the sum to 2^-23.  Where products are alike and of one sign that is 2^-24 of the sum each time;
 * small products beside a large one may be lost whole.  Sums are joined in fp32 from parts of 2048 values for
 * results in fp32 (which lose 2^-18 of alike products, under 1e-6 where signs mix, and never more than 2^-14 +
 * 2^-17 of the magnitudes) and of 65536 for results in bf16 (2^-13, under 2^-9 + 2^-12 always, beside 2^-9 of
 * rounding).  op transposes its argument where the flag is nonzero.  For a layer y = x W^T with x
 * [tokens, in] and W [out, in]:
 *   forward          y  = x  W^T    transpose_b
 *   input gradient   dx = dy W      neither
 *   weight gradient  dW = dy^T x    transpose_a
 * accumulate adds the product to C (gradients over several batches).
 *   workspace   16-byte aligned, at least the bytes that dipaco_packed_matmul_workspace reports for
 *               the product's extents C [m, n], contraction k (a host-only query; may be zero)
 */
int dipaco_packed_matmul_workspace(int64_t m, int64_t n, int64_t k, int64_t *bytes);
int dipaco_packed_matmul(const dipaco_packed *a, const dipaco_packed *b, int32_t transpose_a, int32_t transpose_b,
                         void *c, int64_t c_stride, int32_t dtype, int32_t accumulate, void *workspace,
                         int64_t workspace_bytes, int32_t device, void *cuda_stream);

/*
 * Linear layers on packed matrices: the products above with what surrounds them in a block done on their fp32
 * sums.  x [tokens, in], w [out, in], bias [out] of bias_dtype or NULL.
 *   linear                y = act(x w^T + bias) + residual, rounded once to dtype (that of a residual; NULL = none).
 *                         The sums are those of dipaco_packed_matmul, and so is the workspace (of its query for m =
 *                         tokens, n = out, k = in).
 *   linear_pack           a = x w^T + bias and y = act(a), both packed from their fp32 values: y for the next
 *                         layer, a as the checkpoint that the backward call reads (NULL = not wanted)
 *   linear_pack_backward  da = (dy w) act'(a), packed, for dy [tokens, out] packed and a [tokens, in] as linear_pack
 *                         left it for the layer before (not read without an activation), and dbias = sum of da
 *                         over the tokens, of its fp32 values ([in] fp32, zero for no tokens; NULL = not wanted).
 *                         workspace: of its query for m = tokens, n = in, k = out; only needed for dbias
 * Activations: relu(a) = max(a, 0); silu(a) = a / (1 + exp(-a)); gelu as above.  An infinity of a is NaN once it is
 * packed, and makes silu and gelu NaN or infinite; NaN stays NaN.  relu'(0) = 0.
 * The packed forms refuse contractions over 65536 (DIPACO_ELIMIT).  linear_pack takes its sums in one go, as results
 * in bf16 do; linear_pack_backward those over up to 8192 values (2^-16 of alike products of one sign, which dbias then
 * has lost too), and longer ones in parts of 2048, as results in fp32.
 */
enum {
    DIPACO_ACTIVATION_NONE = 0,
    DIPACO_ACTIVATION_RELU = 1,
    DIPACO_ACTIVATION_SILU = 2,
    DIPACO_ACTIVATION_GELU = 3
};
int dipaco_packed_linear(const dipaco_packed *x, const dipaco_packed *w, const void *bias, int32_t bias_dtype,
                         int32_t activation, const void *residual, int64_t residual_stride, void *y, int64_t y_stride,
                         int32_t dtype, void *workspace, int64_t workspace_bytes, int32_t device, void *cuda_stream);
int dipaco_packed_linear_pack_workspace(int64_t m, int64_t n, int64_t k, int64_t *bytes);
int dipaco_packed_linear_pack(const dipaco_packed *x, const dipaco_packed *w, const void *bias, int32_t bias_dtype,
                              int32_t activation, const dipaco_packed *y, const dipaco_packed *a, void *workspace,
                              int64_t workspace_bytes, int32_t device, void *cuda_stream);
int dipaco_packed_linear_pack_backward_workspace(int64_t m, int64_t n, int64_t k, int64_t *bytes);
int dipaco_packed_linear_pack_backward(const dipaco_packed *dy, const dipaco_packed *w, const dipaco_packed *a,
                                       int32_t activation, const dipaco_packed *da, float *dbias, void *workspace,
                                       int64_t workspace_bytes, int32_t device, void *cuda_stream);

/*
 * The norm of several gradients together, sqrt of the sum of all their squares, and the gradients times
 * min(1, max_norm / norm).  Squares are added in fp32 for at most 80 values (in chains of 20) and in fp64 beyond, or
 * in fp64 where fp32 would overflow or lose them.  Under a limit a norm that is not finite shows: with a NaN all
 * results are NaN, with an infinity they are zero, or NaN where the gradient is infinite.
 *   grads        HOST array [count] of device pointers, gradient i being numel[i] contiguous values of dtypes[i]
 *   out          HOST array of device pointers to as many values of out_dtypes[i]; a result is its own gradient's
 *                tensor (in place, of the same type) or overlaps nothing else; NULL = the norm alone
 *   max_norm     >= 0; infinity = no clipping: results are copies, whatever the norm
 *   norm         fp32, before clipping; may be NULL, and is then not computed for copies
 *   workspace    16-byte aligned, at least the bytes that dipaco_clip_gradients_workspace reports (host only); not
 *                needed for copies without the norm
 * The arrays are read before the call returns.
 */
int dipaco_clip_gradients_workspace(const int64_t *numel, int32_t count, int64_t *bytes);
int dipaco_clip_gradients(const void *const *grads, void *const *out, const int64_t *numel, const int32_t *dtypes,
                          const int32_t *out_dtypes, int32_t count, double max_norm, float *norm, void *workspace,
                          int64_t workspace_bytes, int32_t device, void *cuda_stream);

/*
 * Every wait inside the kernels of this section is bounded (4 s).  A wait that runs out ends its kernel in
 * an orderly way with undefined results; later calls work again.  This call synchronises the stream and
 * returns DIPACO_ETIMEOUT if that has happened on the device, on whatever stream, since it was last called
 * for this stream (or ever, the first time), DIPACO_OK otherwise: no stream takes the news from another.
 */
int dipaco_inner_status(int32_t device, void *cuda_stream);

/*
 * Diagnostic: make a bounded wait of the norms (operators = 0; of the plain ones, then of those around a block), of
 * the packing kernels (1) or of the products and then the linear layers (2) run out on purpose, harmlessly: one warp
 * waits at most limit_ns (1 .. 1e9) on a barrier that nothing will complete; no copy is in flight and no buffer of the
 * caller is involved.
 */
int dipaco_selftest_inner_wait_expiry(int32_t operators, int64_t limit_ns, int32_t device, void *cuda_stream);

const char *dipaco_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* DIPACO_H */
